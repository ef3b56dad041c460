"""Pins of the 4-bit cache's oracle: hand-worked blocks, exhaustive rounding, brute force (no GPU)."""
import itertools

import numpy as np
import pytest

from oracle import kv4_attn_weight_ref, kv4_evict_ref, kv4_quantise_ref, kv4_values_ref


def _block(*values):
    x = np.zeros(32)
    x[:len(values)] = values
    return x


def test_hand_worked_block():
    # largest 7 -> scale 1; 7 -> 6; 5 is a tie between 4 (code 6) and 6 (code 7): 4; 2.5 between 2 (code 4) and 3: 2
    codes, scales = kv4_quantise_ref(_block(7.0, -5.0, 2.5, 0.25, 0.75, -0.74))
    assert scales.tolist() == [127]
    assert codes[:3].tolist() == [7 | (14 << 4), 4 | (0 << 4), 2 | (9 << 4)]
    assert kv4_values_ref(codes, scales)[:6].tolist() == [6.0, -4.0, 2.0, 0.0, 1.0, -0.5]


@pytest.mark.parametrize("top,scale", [(7.0, 127), (7.0001, 128), (3.5, 126), (3.50001, 127), (6.0, 127), (4.0, 127), (0.0, 1), (1e-40, 1),
                                       (3e38, 252)])
def test_scale_is_the_smallest_that_brings_the_largest_to_seven(top, scale):
    assert kv4_quantise_ref(_block(top))[1].tolist() == [scale]


def test_every_element_is_the_nearest_and_values_go_through_unchanged():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((500, 96)) * np.exp2(rng.integers(-20, 20, (500, 1)))
    codes, scales = kv4_quantise_ref(x)
    y = kv4_values_ref(codes, scales)
    unit = np.repeat(np.exp2(scales - 127.0), 32, -1)
    signed = np.concatenate([np.array([0, .5, 1, 1.5, 2, 3, 4, 6]), -np.array([.5, 1, 1.5, 2, 3, 4, 6])])
    far = np.abs(x[..., None] / unit[..., None] - signed).min(-1)
    assert np.allclose(np.abs(x - y) / unit, far, atol=1e-12)
    assert (np.abs(x / unit).reshape(500, 3, 32).max(-1) <= 7).all() and (np.abs(x / unit).reshape(500, 3, 32).max(-1) > 3.5).all()
    # what is representable under a scale of its own comes back, whatever scale it is written under
    again = kv4_values_ref(*kv4_quantise_ref(y))
    assert np.array_equal(again, y)


def test_blocks_that_hold_something_not_finite_are_nan():
    x = np.ones((3, 64))
    x[0, 3], x[1, 40], x[2, 0] = np.inf, np.nan, -np.inf
    y = kv4_values_ref(*kv4_quantise_ref(x))
    assert np.isnan(y[0, :32]).all() and (y[0, 32:] == 1).all()
    assert np.isnan(y[1, 32:]).all() and (y[1, :32] == 1).all()
    assert np.isnan(y[2, :32]).all()


def test_weights_of_one_row_sum_to_its_share():
    rng = np.random.default_rng(1)
    k = rng.standard_normal((3, 2, 4, 8))
    q = rng.standard_normal((2, 4, 8))
    table = np.array([[2, 0, 1]])
    flat = k[table[0]].transpose(0, 2, 1, 3).reshape(12, 2, 8)[:10]
    lse = np.array([[np.log(np.exp(0.3 * flat[:, h // 2] @ q[r, h]).sum()) for h in range(4)] for r in range(2)])
    w = kv4_attn_weight_ref(q, k, table, [10], [[0, 1]], lse, 0.3, 0.5, np.full((1, 2, 12), 2.0))
    assert np.allclose(w[0, :, :10].sum(-1), 0.5 * 2 * 10 + 2 * 2)  # two rows, two heads a group
    assert (w[0, :, 10:] == 2).all()


def test_eviction_by_brute_force_over_small_weights():
    for weight in itertools.product([0.0, 1.0, 2.0], repeat=5):
        for budget in (1, 3, 5, 7):
            kept = kv4_evict_ref(5, budget, 1, 0, 9, weight, [0, 2, 3, 8, 5])  # position 8 is recent
            assert len(kept) == min(budget, 5) and len(set(kept)) == len(kept) and 3 in kept
            gone = set(range(5)) - set(kept)
            assert all((weight[g], -g) < (weight[k], -k) for g in gone for k in kept if k != 3)
            assert all(kept[i] == i for i in range(len(kept)) if i in kept)
            moved = [k for i, k in enumerate(kept) if k != i]
            assert moved == sorted(moved) and all(m >= len(kept) for m in moved)


def test_protected_positions_stay_in_front_of_infinite_weights():
    assert kv4_evict_ref(4, 2, 1, 0, 9, [np.inf, np.inf, 0.5, 2.0], [0, 2, 3, 8]) == [0, 3]
    assert kv4_evict_ref(4, 1, 1, 0, 9, [np.inf, np.inf, 0.5, 2.0], [0, 2, 3, 8]) == [3]
