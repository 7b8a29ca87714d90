"""Selection where a beam's score is so large that sums in 64 bits hold few places of its tokens' logits: tokens that differ have one score, and among
equal scores the lowest row and the lowest token come first.
"""
import math

import numpy as np
import pytest

import beam_reference as ref
from test_gpu_beam_select import Call, xg  # noqa: F401

pytestmark = pytest.mark.gpu


def _far_from_a_border(x, allowed, scores, over_all):
    """Whether every row's score less its sum lies clear of the middle between two neighbours, so that the last places of a sum do not tell."""
    for r, s in enumerate(scores.astype(np.float32).astype(np.float64)):
        ok = np.ones(x.shape[1], dtype=bool) if allowed is None else allowed[r]
        total, _ = ref.log_total(x[r], np.ones(x.shape[1], dtype=bool) if over_all else ok)
        step = math.ulp(abs(s)) / 2                                  # (below a power of two the neighbours lie half as far apart)
        if abs(total / step % 1 - 0.5) < 1e-6 * max(1, 1 / step):
            return False
    return True


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("level", [3e12, -1e13, 1e14, -4e14, 2e15, -2e15])
def test_scores_that_swallow_differences(xg, dtype, level):  # noqa: F811
    rng = np.random.default_rng(int(abs(level) / 1e12))
    tried = 0
    for K, V, n in ((1, 300, 1), (1, 5000, 1), (1, 5000, 3), (2, 5000, 1), (4, 20011, 2), (4, 5000, 40)):
        for mask in (False, True):
            # the best of a row lie close to each other: a tenth of them within a thousandth to a half of the best
            x = (rng.standard_normal((K, V)) * 2).astype(np.float32)
            x[:, rng.choice(V, V // 10, replace=False)] = 9 - rng.random((K, V // 10)).astype(np.float32) * rng.choice([0.004, 0.06, 0.5], (K, 1)).astype(np.float32)
            allowed = rng.random((K, V)) < 0.8 if mask else None
            scores = np.full(K, level)
            if dtype == "bf16":
                x = ref.from_bf16(ref.to_bf16(x))
            if not _far_from_a_border(x, allowed, scores, mask):
                continue
            tried += 1
            Call(xg, x, allowed, scores, None, 1, K, n, mask, dtype).check((K, V, n, mask))
    assert tried >= 6
