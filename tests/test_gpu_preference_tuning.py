"""The operators together, as examples/preference_tuning.py uses them."""
import importlib.util
import math
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_example(dtype):
    spec = importlib.util.spec_from_file_location("preference_tuning", os.path.join(ROOT, "examples", "preference_tuning.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, off = example.main(steps=8, dtype=dtype, say=lambda s: None)
    # the policy starts as its reference: every ratio is 0 and the loss log 2 (in bfloat16 the reference is the same logits' too)
    assert abs(losses[0] - math.log(2)) <= 1e-4
    assert losses[-1] < losses[0] - 0.05 and all(math.isfinite(x) for x in losses)
    # rows one by one against caches and all rows at once: the same sums in another order, on logits of size 3
    assert off <= (1e-4 if dtype == "fp32" else 0.15)
