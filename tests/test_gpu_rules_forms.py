"""GPU tests of the rules at the largest vocabulary."""
import numpy as np
import pytest
import torch

from test_gpu_rules import _TYPES, _check, _rules, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind,in_place,pad", [("f32", False, 0), ("f32", True, 0), ("bf16", False, 3), ("f16", True, 1)])
def test_the_largest_vocabulary(kind, in_place, pad):
    rng = np.random.default_rng(21)
    B, R, V = 2, 2, 1 << 20
    x = torch.from_numpy(rng.standard_normal((B, R, V)).astype(np.float32) * 4).to(_TYPES[kind][0])
    rules = _rules(rng, B, R, V, hist=900)
    rules["history"][:, -40:] = V - 1 - np.arange(40)
    rules["history_lens"][:] = 900
    rules["mask_rows"][:] = [[-1, 0], [3, 2]]
    tokens = rng.integers(V - 8200, V, (B, R)).astype(np.int32)
    _check(x, _run(x, rules, tokens, None, kind, pad, 0, in_place), kind, rules, tokens, None)
