import functools
import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a real MI355X (run with -m gpu)")


# Tests that hold one wall-clock time against another run behind all the others: with -x the run ends where a clock has changed under one
# of them, and nothing else is hidden by it.  Those that look at nothing but times are measured again where one is too long, twice at
# most: the closest of their bounds, 1.12, is met with 4 % to spare on a quiet device (1.066 to 1.085 in eight measurements).
TIMES_ALONE = {"test_finalising_few_candidates_takes_less_than_many", "test_seventeen_tokens_take_hardly_longer_than_sixteen",
               "test_128_rows_take_hardly_longer_than_64_on_few_vocabulary_tiles"}
TIMED = TIMES_ALONE | {"test_topk_takes_no_longer_for_a_common_offset", "test_topk_takes_no_longer_for_scattered_masks"}


def _measured_again(test):
    @functools.wraps(test)
    def run(*args, **kwargs):
        for _ in range(2):
            try:
                return test(*args, **kwargs)
            except AssertionError as e:
                print(f"measured again: {e}")
        return test(*args, **kwargs)
    return run


def pytest_collection_modifyitems(config, items):
    name = lambda item: getattr(item, "originalname", None)
    for item in items:
        if name(item) in TIMES_ALONE:
            item.obj = _measured_again(item.obj)
    items.sort(key=lambda item: name(item) in TIMED)
    # GPU tests never run by accident on a machine without a device
    try:
        import torch
        have_gpu = torch.cuda.is_available()
    except Exception:  # pragma: no cover
        have_gpu = False
    if have_gpu:
        return
    skip = pytest.mark.skip(reason="no GPU in this process")
    for item in items:
        if "gpu" in item.keywords:
            item.add_marker(skip)
