"""Selection where logits are signalling NaN: no candidate and not counted, like any other NaN.  Arithmetic makes quiet ones only, so these bits
come from outside (a buffer that was never written, a cast of integers); of two operands of a maximum they take the number away.
"""
import numpy as np
import pytest

from test_gpu_beam_select import Call, _inputs, xg  # noqa: F401

pytestmark = pytest.mark.gpu

SIGNALLING = {"f32": [0x7F800001, 0x7FBFFFFF, 0xFF800001, 0xFFA00000], "bf16": [0x7F81, 0x7FBF, 0xFF81, 0xFFA0]}


def _call(xg, rng, x, allowed, scores, G, K, n, over_all, dtype, **kw):  # noqa: F811
    """A call whose NaN, those of the padding too, are signalling."""
    import torch
    c = Call(xg, x, allowed, scores, None, G, K, n, over_all, dtype, **kw)
    bits = c.logits.view(torch.int32) if dtype == "f32" else c.logits
    raw = bits.cpu().numpy().view(np.uint32 if dtype == "f32" else np.uint16).copy()
    nan = (raw & (0x7FFFFFFF if dtype == "f32" else 0x7FFF)) > (0x7F800000 if dtype == "f32" else 0x7F80)
    assert nan.any()
    raw[nan] = rng.choice(np.array(SIGNALLING[dtype], dtype=raw.dtype), nan.sum())
    bits.copy_(torch.from_numpy(raw.view(np.int32 if dtype == "f32" else np.int16)))
    return c


MASKS = [("none", False), ("all", False), ("all", True), ("most", False), ("most", True)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mask,over_all", MASKS)
@pytest.mark.parametrize("V", [2, 3, 33, 300, 2048, 5003])
def test_one_number_beside_them(xg, dtype, mask, over_all, V):  # noqa: F811
    """One finite logit, signalling NaN in some or all of the other places, minus infinity in the rest; the number at every place of a vector."""
    rng = np.random.default_rng(V)
    K = 18
    x = np.full((K, V), -np.inf, dtype=np.float32)
    allowed = None if mask == "none" else np.ones((K, V), dtype=bool)
    for k in range(K):
        at = k % V if k < 9 else int(rng.integers(0, V))
        if mask == "most":
            allowed[k] = rng.random(V) < 0.7
        near = np.arange(max(0, at - 8), min(V, at + 9))
        if k % 3 == 0:
            x[k] = np.nan                                            # everywhere
        elif k % 3 == 1:
            x[k, near] = np.nan                                      # all around
        else:
            x[k, rng.choice(near, 4)] = np.nan                       # here and there
        x[k, at] = 100 - 3 * k
        if allowed is not None:
            allowed[k, at] = True
    x[0, 1] = np.nan                                                 # (row 0 has one in any case)
    scores = -rng.random(K) - 1
    _call(xg, rng, x, allowed, scores, 1, K, K + 2, over_all, dtype, offset=V % 3, pad=2).check((V, mask))
    for k in range(K):
        _call(xg, rng, x[k:k + 1], None if allowed is None else allowed[k:k + 1], scores[k:k + 1], 1, 1, 2, over_all, dtype, offset=k, pad=1).check((V, mask, k))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_piece_that_has_one_number(xg, dtype):  # noqa: F811
    """Rows of many pieces, of which one has a single finite logit among signalling NaN and minus infinity: the row's best, or one that
    counts in its sum."""
    rng = np.random.default_rng(6)
    V = 3 * 2048 + 700
    for mask, over_all in MASKS:
        x = (rng.standard_normal((8, V)) * 2).astype(np.float32)
        allowed = None if mask == "none" else np.ones((8, V), dtype=bool) if mask == "all" else rng.random((8, V)) < 0.7
        for k in range(8):
            lo = 2048 * (k % 3)
            x[k, lo:lo + 2048] = np.nan if k % 2 else -np.inf
            at = lo + int(rng.integers(40, 2000))
            x[k, at - 8:at + 9] = np.nan
            x[k, at] = 12 if k < 4 else 7
            if allowed is not None:
                allowed[k, at] = True
        scores = -rng.random(8) - 1
        for K, offset in ((1, 0), (4, 0), (8, 5)):
            _call(xg, rng, x, allowed, scores, 8 // K, K, 12, over_all, dtype, offset=offset, pad=3).check((mask, over_all, K))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_among_ordinary_logits(xg, dtype):  # noqa: F811
    """A few of them, many, and nothing else; in places that the mask takes away too."""
    rng = np.random.default_rng(7)
    G, K = 2, 4
    for V in (7, 500, 9001):
        for share in (0.01, 0.5, 0.97, 1.0):
            for mask, over_all in (("none", False), ("mixed", False), ("mixed", True), ("few", False), ("half", True)):
                x, allowed, scores, _ = _inputs(rng, G, K, V, mask)
                x[rng.random((G * K, V)) < share] = np.nan
                x[0, 0] = np.nan
                _call(xg, rng, x, allowed, scores, G, K, 9, over_all, dtype, pad=1).check((V, share, mask, over_all))
