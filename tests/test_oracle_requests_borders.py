"""Pins of the oracle of sampling rules and pages at their borders (no GPU)."""
import numpy as np

from oracle import rules_logits_ref


def test_a_penalty_falls_on_what_was_there():
    inf = float("inf")
    counts = np.array([[0, 2, 1 << 30]])
    for presence, frequency in ((inf, 0.0), (0.0, inf), (float("nan"), 0.5)):
        z = rules_logits_ref([[1.0, 2.0, 4.0]], [0, 1], None, None, counts, [[1.0, 2.0, presence, frequency]], [[(0, 0.5)]], None, None)
        assert z.tolist() == [[1.5, -inf, 2.0]]
