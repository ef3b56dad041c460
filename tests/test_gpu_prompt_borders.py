"""hb_prompt_attn where weights and values come near the ends of float32: results that are finite are found, and rows beside them
keep their bits."""
import numpy as np
import pytest
import torch

import workloads as W
from prompts import Prompts
from test_gpu_prompt_attn import _algos

pytestmark = pytest.mark.gpu


def _along_one_dimension(c, scores):
    """Every row's natural score of prefix position p is scores[p], of prompt row i scores[len + i] (one sequence)."""
    c.scale = 0.125
    c.q[:], c.k[:] = 0, 0
    c.q[:, :, 0] = 8.0
    n = c.lens[0]
    for p in range(n):
        c.k_pool[c.table[0, p // c.page], :, p % c.page] = 0
        c.k_pool[c.table[0, p // c.page], :, p % c.page, 0] = scores[p]
    c.k[:, :, 0] = torch.tensor(scores[n:], dtype=c.tdtype)[:, None]


def _value(c, p, x):
    """The values of position p (prefix, then prompt rows)."""
    n = c.lens[0]
    if p < n:
        c.v_pool[c.table[0, p // c.page], :, p % c.page] = x
    else:
        c.v[p - n] = x


def _large(D, key, score, sizes):
    """Rows behind ``key`` see a value of ``sizes`` (one a dimension, over and over) whose score is the only one above 0."""
    def make(dtype):
        c = Prompts(41, dtype, 4, 2, D, 16, [70], [300])
        scores = [0.0] * 370
        scores[key] = score
        _along_one_dimension(c, scores)
        _value(c, key, torch.tensor(np.resize(sizes, D), dtype=c.tdtype))
        return c
    return make


# A key of a later block whose score is 7 to 8 in base 2 above the first one's: it takes a quarter to two thirds of a row
CASES = {
    "prefix, 64": _large(64, 40, 4.84375, [3.0e38, -3.0e38, 1.0, 1e-3]),
    "prefix, 128": _large(128, 66, 5.5, [-3.0e38, 2.0, 3.0e38]),
    "prompt, 64": _large(64, 150, 5.5, [3.0e38]),
    "prompt, 128": _large(128, 200, 4.84375, [2.0e36, -5.0, 1e37]),
}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", CASES)
def test_a_large_value_with_a_weight_above_the_reference(name, dtype):
    c = CASES[name](dtype)
    ref = c.reference()
    assert np.isfinite(ref[0]).all() and np.abs(ref[0]).max() > 1e35
    for algo in _algos(dtype, c.D, 16):
        for splits in (1, 2, 5):
            out, lse = c.run(algo=algo, num_splits=splits)
            _within(c, out, lse, ref, f"{name} {algo} {splits}")


def _within(c, out, lse, ref, label):
    """As Prompts.check, dimension by dimension, where values differ by forty orders of magnitude.
    Scores here are exact: one product each, of numbers of a few bits.  A weight is off by two roundings of its exponent's argument
    (of at most 16: 2^-20 each) and one of its own, 2^-24; in bf16 by 2^-8 / 2, in the product and the sum, which each takes for
    itself; n of them are added with 2^-24 of the mass each."""
    mass, _ = c.reference(v=np.abs(W.widen(c.v)), v_pool=np.abs(W.widen(c.v_pool)))
    n = c.lens[0] + c.rows[0]
    half = 2.0 ** -24 if c.dtype == "f32" else 2.0 ** -8
    tol = (2 * 3 * 2.0 ** -20 + (n + 16) * 2.0 ** -24) * mass + (half if c.dtype == "bf16" else 0) * mass + 2 * half * np.abs(ref[0]) + 1e-30
    got = W.widen(out)
    assert np.isfinite(got).all(), (label, np.argwhere(~np.isfinite(got))[:3])
    assert (np.abs(got - ref[0]) <= tol).all(), (label, (np.abs(got - ref[0]) / tol).max())
    assert np.abs(W.widen(lse) - ref[1]).max() <= 3 * 2.0 ** -20 + (n + 16) * 2.0 ** -24 + 2.0 ** -22 * np.abs(ref[1]).max(), label


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("low", [-86.0, -87.5, -89.0, -95.0, -104.0])
def test_small_scores_behind_a_block_of_none(dtype, low):
    """The first 70 keys have scores of -infinity, those behind lie where 2^x leaves float32's normal numbers, some on either side."""
    c = Prompts(44, dtype, 4, 2, 64, 16, [40], [160])
    scores = [-float("inf")] * 70 + [low - (p * 7 % 5) * 0.5 for p in range(130)]
    _along_one_dimension(c, [max(s, -1e30) for s in scores])
    c.k[:30, :, 0], c.k_pool[:, :, :, 0] = -torch.inf, -torch.inf
    c.k[:30, :, 1:], c.q[:, :, 1:] = 0, 0
    with np.errstate(invalid="ignore", divide="ignore"):  # rows that see no other score have no result
        ref, ref_lse = c.reference()
    seen = np.arange(160) >= 30
    # scores are exact; the argument of an exponential is one of (score - reference), off by 2^-17 of scores of up to 128 in float32
    tol = (2.0 ** -14 if dtype == "f32" else 2.0 ** -7) * (np.abs(ref[seen]).max() + 4)
    for algo in _algos(dtype, 64, 16):
        for splits in (1, 2, 3):
            out, lse = c.run(algo=algo, num_splits=splits)
            o = W.widen(out)
            assert np.isnan(o[~seen]).all()
            assert np.abs(o[seen] - ref[seen]).max() <= tol, (algo, splits, np.abs(o[seen] - ref[seen]).max())
            assert np.abs(W.widen(lse)[seen] - ref_lse[seen]).max() <= 1e-4


@pytest.mark.parametrize("dtype,largest", [("f32", 3.0e38), ("bf16", 3.3895313892515355e38)])
@pytest.mark.parametrize("D", [64, 72, 128])
def test_all_values_are_the_types_largest(dtype, largest, D):
    """A mean of such values is such a value, with other signs in every dimension, whole and in parts."""
    c = Prompts(42, dtype, 4, 2, D, 16, [90], [200])
    sign = torch.where(torch.arange(D) % 3 == 0, -1.0, 1.0)
    for p in range(290):
        _value(c, p, (largest * sign).to(c.tdtype))
    for algo in _algos(dtype, D, 16):
        for splits in (1, 2, 4):
            out, _ = c.run(algo=algo, num_splits=splits)
            # weights of 290 keys and their sum: (290 + 16) 2^-24 twice; in bf16 less than the half step that they are rounded to
            far = np.abs(W.widen(out) / (largest * sign.double().numpy()) - 1)
            assert far.max() <= (2 * 306 * 2.0 ** -24 if dtype == "f32" else 0), (algo, splits, far.max())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_that_do_not_see_a_large_value_keep_their_bits(dtype):
    """The same workgroup has rows whose sums overflow at first and rows whose do not."""
    c = Prompts(43, dtype, 4, 2, 64, 16, [20], [120], sharp=2.0)
    for algo in _algos(dtype, 64, 16):
        for splits in (1, 3):
            want, want_lse = c.run(algo=algo, num_splits=splits)
            d = c.device()
            d["v"][50:] = 3.3e38
            d["v"][90, 0, 3] = torch.inf
            got, got_lse = c.run(dev=d, algo=algo, num_splits=splits)
            assert torch.equal(got[:50], want[:50]) and torch.equal(got_lse[:50], want_lse[:50])
            assert torch.equal(got_lse[:50], want_lse[:50]) and torch.isfinite(got[50:90].float()).all()
            assert (got[90:, :2, 3] == torch.inf).all() and torch.isfinite(got[90:, 2:].float()).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 136])
def test_many_parts_of_large_values(dtype, D):
    """More parts than a thread of the join has, each with a finite result of its own near the type's largest, whose sum is beyond it."""
    c = Prompts(45, dtype, 4, 2, D, 16, [5000], [3])
    for p in range(5003):
        _value(c, p, 3.0e38)
    exact = float(torch.tensor(3.0e38, dtype=c.tdtype).double())
    for algo in _algos(dtype, D, 16):
        for splits in (0, 18, 70):
            out, _ = c.run(algo=algo, num_splits=splits)
            far = np.abs(W.widen(out) / exact - 1)
            # sums of 5003 weights and as many products, 2^-24 each at most
            assert far.max() <= (2 * 5100 * 2.0 ** -24 if dtype == "f32" else 2.0 ** -8), (algo, splits, far.max())
