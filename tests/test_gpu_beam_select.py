"""Selection over beams and vocabulary against the definition in 64 bits: parents, tokens and whether they have ended exactly, scores
within the tolerance derived in beam_reference.
"""
import numpy as np
import pytest

import beam_reference as ref
import oracle

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def xg():
    import torch
    assert torch.cuda.is_available()
    import paper_2601_04426_amd as xg
    return xg


def _stream():
    import torch
    return torch.cuda.current_stream().cuda_stream


def _put(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


class Call:
    """One call with everything around it: rows at `offset` elements, `pad` elements between them (NaN), outputs between guards."""

    def __init__(self, xg, x, allowed, scores, finished, G, K, n, over_all, dtype, eos=0, offset=0, pad=0, mask_pad=0):
        import torch
        self.xg, self.G, self.K, self.n, self.over_all, self.eos = xg, G, K, n, over_all, eos
        R, V = x.shape
        self.V, stride = V, V + pad
        raw = np.full(offset + R * stride + 64, np.nan, dtype=np.float32)
        raw[offset:offset + R * stride].reshape(R, stride)[:, :V] = x
        if dtype == "bf16":
            raw = ref.to_bf16(raw)
        self.x = (ref.from_bf16(raw) if dtype == "bf16" else raw)[offset:offset + R * stride].reshape(R, stride)[:, :V].copy()
        self.logits = _put(raw.view(np.int16) if dtype == "bf16" else raw)
        self.at, self.stride, self.code = self.logits.data_ptr() + offset * raw.itemsize, stride, xg.XG2_BF16 if dtype == "bf16" else xg.XG2_F32
        self.allowed, self.mask, self.mask_stride = allowed, None, 0
        if allowed is not None:
            W = (V + 31) // 32
            words = np.full((R, W + mask_pad), -1, dtype=np.int32)   # (what lies behind a row's words allows everything)
            words[:, :W] = np.stack([oracle.pack_bitmask(a) for a in allowed])
            if V % 32:                                               # and so do the bits behind the last token
                words[:, W - 1] |= np.uint32((0xFFFFFFFF << (V % 32)) & 0xFFFFFFFF).astype(np.int32)
            self.mask, self.mask_stride = _put(words), W + mask_pad
        self.scores, self.finished = scores.astype(np.float32), finished
        self.d_scores, self.d_finished = _put(self.scores), None if finished is None else _put(finished.astype(np.int32))
        self.size = xg.beam_select_workspace(self.code, G, K, V, n)
        self.work = torch.full((self.size + 64,), 0x5A, dtype=torch.uint8, device="cuda")
        self.out = [torch.full((G * n + 8,), 77, dtype=t, device="cuda") for t in (torch.float32, torch.int32, torch.int32, torch.int32)]

    def run(self):
        o = [t.data_ptr() + 16 for t in self.out]
        self.xg.beam_select(self.at, self.code, self.G, self.K, self.V, self.stride, self.d_scores.data_ptr(), self.n, o[0], o[1], o[2], self.work.data_ptr(), self.size,
                            bitmask_ptr=0 if self.mask is None else self.mask.data_ptr(), bm_row_stride_words=self.mask_stride,
                            over=self.xg.XG2_OVER_ALL if self.over_all else self.xg.XG2_OVER_ALLOWED,
                            finished_ptr=0 if self.d_finished is None else self.d_finished.data_ptr(), eos_id=self.eos, out_finished_ptr=o[3], stream=_stream())

    def outputs(self):
        import torch
        torch.cuda.synchronize()
        got = [t.cpu().numpy() for t in self.out]
        assert all((g[:4] == 77).all() and (g[-4:] == 77).all() for g in got), "written beside the outputs"
        assert bool((self.work[self.size:] == 0x5A).all()), "written behind the workspace"
        return [g[4:-4].reshape(self.G, self.n) for g in got]

    def check(self, what=""):
        self.run()
        got = self.outputs()
        want = ref.select(self.x, self.allowed, self.scores, self.finished, self.G, self.K, self.n, self.over_all, self.eos)
        for name, a, b in zip(("parents", "tokens", "finished"), got[1:], want[1:]):
            assert np.array_equal(a, b), (what, name, np.argwhere(a != b)[:4].tolist(), a[a != b][:4], b[a != b][:4])
        none = np.isneginf(want[0])
        assert np.array_equal(np.isneginf(got[0]), none), what
        err = np.abs(got[0][~none].astype(np.float64) - want[0][~none])
        assert (err <= ref.score_tolerance(self.V, want[0][~none])).all(), (what, err.max())
        return got


def _inputs(rng, G, K, V, mask):
    R = G * K
    x = (rng.standard_normal((R, V)) * 2).astype(np.float32)
    x[np.arange(R)[:, None], rng.integers(0, V, (R, 5))] += rng.random((R, 5)).astype(np.float32) * 8
    density = {"none": None, "dense": 0.98, "half": 0.5, "few": 4.0 / V, "empty": 0.0}
    allowed = None
    if mask == "mixed":
        allowed = rng.random((R, V)) < rng.choice([0.99, 0.6, 0.01, 0.0], (R, 1))
    elif mask != "none":
        allowed = rng.random((R, V)) < density[mask]
    scores = -rng.random(R) * 5 - 3
    finished = (rng.random(R) < 0.1).astype(np.int32)
    scores[rng.random(R) < 0.1] = -np.inf
    return x, allowed, scores, finished


# V: within a vector, a mask word, a block of 256 tokens, a piece of 2,048 and around them; rows begin at any place in a line
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 7, 31, 32, 33, 255, 256, 257, 1985, 2047, 2048, 2049, 2111, 4097, 8192, 50021])
def test_rows_at_any_place(xg, dtype, V):
    rng = np.random.default_rng(V)
    for k, (mask, over_all, offset, pad) in enumerate([("none", False, 0, 0), ("mixed", False, 1, 1), ("mixed", True, 3, 0), ("half", False, 31, 7), ("few", True, 63, 64), ("dense", True, 5, 3),
                                                       ("few", False, 64, 0), ("empty", False, 2, 5), ("empty", True, 0, 1)]):
        G, K, n = [(2, 3, 5), (1, 4, 8), (3, 1, 2), (1, 8, 16)][k % 4]
        x, allowed, scores, finished = _inputs(rng, G, K, V, mask)
        Call(xg, x, allowed, scores, finished if k % 2 else None, G, K, n, over_all, dtype, eos=V // 2, offset=offset, pad=pad, mask_pad=k % 3).check((V, mask, over_all, offset, pad))


@pytest.mark.parametrize("G,K,n", [(1, 1, 1), (5, 1, 128), (1, 64, 128), (2, 64, 64), (3, 17, 33), (70, 2, 3), (1, 33, 1), (4, 16, 16)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_groups_and_candidates(xg, dtype, G, K, n):
    rng = np.random.default_rng(G * 100 + K)
    for V, mask, over_all in ((3000, "mixed", False), (700, "none", False), (40, "half", True), (3, "none", True)):
        x, allowed, scores, finished = _inputs(rng, G, K, V, mask)
        Call(xg, x, allowed, scores, finished, G, K, n, over_all, dtype).check((V, mask))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("K,V,n", [(1, 60, 128), (1, 500, 16), (1, 5000, 128), (2, 129, 128), (4, 2000, 8), (4, 300, 100), (8, 8000, 16), (32, 2000, 32), (64, 100, 128), (3, 70000, 128)])
def test_rows_that_differ_and_few_pieces(xg, dtype, K, V, n):
    """Rows from nearly everything allowed to a handful, and fewer pieces or blocks of the vocabulary than candidates wanted."""
    rng = np.random.default_rng(K * 1000 + V)
    G = 3
    x, allowed, scores, finished = _inputs(rng, G, K, V, "mixed")
    for over_all in (False, True):
        Call(xg, x, allowed, scores, finished, G, K, n, over_all, dtype).check(over_all)
    x[::2] -= 6                                                      # every other beam is far behind in all it has
    Call(xg, x, None, scores, finished, G, K, n, False, dtype).check("behind")


def test_large_magnitudes(xg):
    """Logits and scores whose exponentials or sums a row's first pass cannot take."""
    rng = np.random.default_rng(10)
    K, V = 6, 5000
    x = (rng.standard_normal((K, V)) * 2).astype(np.float32)
    x[1] *= 1e5
    x[2] = x[2] * 1e30
    x[3] += 3e6
    x[4] -= 2e9
    x[5, 10:] -= 1e9
    for scores in (np.full(K, -1.0), np.array([-1.0, -2e5, -3e30, -4e6, 5e6, -6.0]), np.array([2e15, 2e15, 2e15, 1e30, 1e30, -1e30])):
        for dtype in ("f32", "bf16"):
            Call(xg, x, None, scores, None, 1, K, 40, False, dtype).check(scores)
            Call(xg, x, rng.random((K, V)) < 0.5, scores, None, 2, 3, 40, True, dtype).check(scores)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_logits_that_are_alike(xg, dtype):
    """Ties go to the lowest row, then to the lowest token: all logits the same, a handful of values, the same rows again."""
    rng = np.random.default_rng(5)
    G, K, V = 2, 4, 6000
    R = G * K
    zeros = np.zeros((R, V), dtype=np.float32)
    few = rng.integers(-2, 3, (R, V)).astype(np.float32)
    same = np.repeat((rng.standard_normal((G, 1, V)) * 2).astype(np.float32), K, 1).reshape(R, V)
    flat = np.full(R, -1.5)
    for name, x in (("zeros", zeros), ("few", few), ("same", same)):
        for scores in (flat, np.linspace(-1, -2, R)):
            for n in (1, 7, 128):
                for allowed in (None, np.repeat(rng.random((1, V)) < 0.5, R, 0)):
                    Call(xg, x, allowed, scores, np.zeros(R), G, K, n, False, dtype).check((name, n))
    # nearly every block has the same best token (more than the kernel's lists take), with beams that have ended among them
    x = np.full((64, 9000), -3.0, dtype=np.float32)
    x[:, ::100] = 2.0
    finished = (np.arange(64) % 5 == 0).astype(np.int32)
    Call(xg, x, None, np.full(64, -8.0), finished, 1, 64, 128, False, dtype).check("blocks alike")
    Call(xg, x, None, np.full(64, -8.0), finished, 2, 32, 100, True, dtype).check("blocks alike")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_closer_than_a_sum_in_32_bits(xg, dtype):
    """The same logits in another order: the rows' candidates differ by what their scores differ, far less than a sum in 32 bits is
    off (the logits are, as beams of one prompt have them, not small)."""
    rng = np.random.default_rng(9)
    for trial in range(8):
        V = int(rng.integers(2000, 20000))
        base = (rng.standard_normal(V) * 3 + 20).astype(np.float32)
        base[rng.integers(0, V, 40)] += 6
        x = np.stack([rng.permutation(base) for _ in range(4)])
        scores = rng.permutation(np.array([0.0, 3e-9, -2e-9, 7e-9]))
        Call(xg, x, None, scores, None, 1, 4, 32, False, dtype).check(trial)
        Call(xg, x, np.ones((4, V), dtype=bool), scores, None, 2, 2, 16, True, dtype).check(trial)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("over_all", [False, True])
def test_infinities_and_nan(xg, dtype, over_all):
    rng = np.random.default_rng(11)
    G, K, V, n = 2, 8, 5000, 20
    R = G * K
    low = float(np.finfo(np.float32).min) if dtype == "f32" else float(ref.from_bf16(np.array([0xFF7F], dtype=np.uint16))[0])
    x, allowed, scores, finished = _inputs(rng, G, K, V, "mixed")
    scores[:] = -np.linspace(2, 3, R)
    allowed[0], allowed[1] = False, False
    x[1] = np.nan                                                    # nothing but NaN, nothing allowed
    x[2, rng.random(V) < 0.3] = np.nan
    allowed[3] = rng.random(V) < 0.5
    x[3, ~allowed[3]] = rng.choice(np.array([np.nan, np.inf, -np.inf, low], dtype=np.float32), (~allowed[3]).sum())   # in masked places
    x[4, rng.integers(0, V, 3)] = np.inf
    allowed[4] |= np.isposinf(x[4])
    x[5], allowed[5] = low, rng.random(V) < 0.01                     # a mask of the type's lowest value, and nothing else
    x[6, 100:] = low
    x[7, 50:] = -np.inf
    x[8] = -np.inf
    x[9, :] = low
    x[9, 77] = 0.5
    x[10] = -low                                                     # the largest finite value
    x[11, ::2] = np.nan
    x[12, 0], x[13, V - 1] = np.inf, np.nan
    for mask in (allowed, None):
        Call(xg, x, mask, scores, None, G, K, n, over_all, dtype).check("rows of all kinds")
    for r in range(R):                                               # and each kind by itself
        Call(xg, x[r:r + 1], allowed[r:r + 1], scores[r:r + 1], None, 1, 1, n, over_all, dtype).check(r)


def test_beams_that_are_none(xg):
    rng = np.random.default_rng(12)
    G, K, V = 3, 6, 900
    x, _, _, _ = _inputs(rng, G, K, V, "none")
    scores = np.array([-1, -np.inf, np.nan, np.inf, -2, -3] + [-np.inf] * 6 + [-5, -5, -5, -np.inf, -1, -1], dtype=np.float64)
    finished = np.array([0, 1, 1, 1, 1, 0] + [1, 0] * 3 + [1, 1, 0, 1, 7, -1])
    x[1] = np.nan
    got = Call(xg, x, None, scores, finished, G, K, 9, False, "f32").check()
    assert (got[1][1] == -1).all() and (got[3][1] == 1).all()        # a group without beams
    Call(xg, x, np.zeros((G * K, V), dtype=bool), scores, finished, G, K, 9, False, "f32").check()


def test_no_outputs_for_finished(xg):
    rng = np.random.default_rng(13)
    x, allowed, scores, _ = _inputs(rng, 1, 4, 500, "half")
    c = Call(xg, x, allowed, scores, None, 1, 4, 4, False, "f32")
    o = [t.data_ptr() + 16 for t in c.out]
    xg.beam_select(c.at, c.code, 1, 4, 500, c.stride, c.d_scores.data_ptr(), 4, o[0], o[1], o[2], c.work.data_ptr(), c.size, bitmask_ptr=c.mask.data_ptr(),
                   bm_row_stride_words=c.mask_stride, stream=_stream())
    assert (c.outputs()[3] == 77).all()


def test_large_vocabulary_and_many_rows(xg):
    """Masked ends of a row beyond 2^20 tokens; rows beyond a launch's 65,535."""
    import torch
    V = (1 << 20) + 77
    rng = np.random.default_rng(14)
    x = rng.standard_normal((2, V)).astype(np.float32)
    allowed = np.zeros((2, V), dtype=bool)
    allowed[0, [0, V - 1, 1 << 19]] = True
    allowed[1, V - 40:] = True
    for dtype in ("f32", "bf16"):
        Call(xg, x, allowed, np.array([-1.0, -2.0]), None, 1, 2, 50, False, dtype).check()
        Call(xg, x, None, np.array([-1.0, -2.0]), None, 1, 2, 50, False, dtype).check()
    G, K, V = 70001, 1, 40
    x = rng.standard_normal((G, V)).astype(np.float32)
    Call(xg, x, None, np.full(G, -1.0), None, G, K, 2, False, "bf16").check()
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_logits_nearly_the_same(xg, dtype):
    """All tokens as far from their beams as the others: from logits that differ by tenths to those that differ in their last bits."""
    rng = np.random.default_rng(21)
    for k, (G, K, V, n) in enumerate([(1, 4, 9000, 8), (2, 16, 20011, 64), (1, 64, 3001, 128), (3, 2, 50021, 1)]):
        for spread, level in ((0.3, 0.0), (0.03, 0.0), (1e-3, 5.0), (1e-5, -2.0)):
            x = (rng.standard_normal((G * K, V)) * spread + level).astype(np.float32)
            scores = -rng.random(G * K) * (4 * spread if k % 2 else 2.0) - 1
            finished = (rng.random(G * K) < 0.1).astype(np.int32)
            allowed = rng.random((G * K, V)) < 0.9 if k % 2 else None
            Call(xg, x, allowed, scores, finished, G, K, n, bool(k & 2), dtype).check((G, K, V, n, spread))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masks_of_few_tokens_a_word(xg, dtype):
    """Words that allow one, six and seven tokens, at a row's ends too; NaN and infinities among them and beside them."""
    rng = np.random.default_rng(24)
    for V in (31, 200, 2048, 5003):
        for most in (1, 3, 6, 7):
            x = (rng.standard_normal((6, V)) * 2).astype(np.float32)
            allowed = np.zeros((6, V), dtype=bool)
            for r in range(6):
                for w in range(0, V, 32):
                    n = min(32, V - w)
                    allowed[r, w + rng.choice(n, min(n, most if rng.random() < 0.3 else rng.integers(0, most + 1)), replace=False)] = True
            allowed[0, [0, V - 1]] = True
            odd = rng.random((6, V)) < 0.05
            x[odd] = rng.choice(np.array([np.nan, -np.inf], dtype=np.float32), odd.sum())
            x[3] = np.where(allowed[3], np.nan, x[3])                # (nothing but NaN)
            x[4, np.flatnonzero(allowed[4])[:2]] = np.inf
            x[5] = np.where(allowed[5], x[5], np.nan)
            scores = -rng.random(6) - 1
            for K, offset in ((1, 0), (3, 1), (6, 3)):
                Call(xg, x, allowed, scores, None, 6 // K, K, 10, False, dtype, offset=offset, pad=7).check((V, most, K))


def test_one_workspace_for_calls_in_a_row(xg):
    """Calls of other sizes, types and masks, one behind the other in a stream, take turns in one workspace."""
    import torch
    rng = np.random.default_rng(22)
    calls = [Call(xg, *_inputs(rng, G, K, V, mask), G, K, n, over, dtype, pad=5)
             for G, K, V, n, mask, over, dtype in ((4, 8, 30011, 16, "mixed", False, "bf16"), (1, 3, 500, 4, "empty", False, "f32"), (2, 32, 7000, 64, "few", True, "f32"), (9, 5, 2100, 9, "none", True, "bf16"))]
    work = torch.full((max(c.size for c in calls) + 64,), 0x5A, dtype=torch.uint8, device="cuda")
    for c in calls:
        c.work = work
    for _ in range(3):
        for c in calls:
            c.run()
    biggest = max(c.size for c in calls)
    for c in calls:
        c.size = biggest                                             # (what lies behind a smaller call's part belongs to the others)
        got = c.outputs()
        want = ref.select(c.x, c.allowed, c.scores, c.finished, c.G, c.K, c.n, c.over_all, c.eos)
        assert all(np.array_equal(g, w) for g, w in zip(got[1:], want[1:]))


def test_logits_and_masks_beyond_4_gib(xg):
    """Rows 3 GB apart, their masks 1.4 GB apart."""
    import torch
    K, V, stride, words = 3, 5003, 1_500_000_019, 350_000_000
    rng = np.random.default_rng(23)
    x = ref.to_bf16((rng.standard_normal((K, V)) * 2).astype(np.float32))
    allowed = rng.random((K, V)) < 0.5
    scores = np.array([-1.0, -1.5, -0.5], dtype=np.float32)
    logits, mask = torch.empty(2 * stride + V, dtype=torch.int16, device="cuda"), torch.empty(2 * words + (V + 31) // 32, dtype=torch.int32, device="cuda")
    for k in range(K):
        logits[k * stride:k * stride + V] = _put(x[k].view(np.int16))
        mask[k * words:k * words + (V + 31) // 32] = _put(oracle.pack_bitmask(allowed[k]))
    n = 40
    o = [torch.empty(n, dtype=t, device="cuda") for t in (torch.float32, torch.int32, torch.int32, torch.int32)]
    d_scores = _put(scores)
    work = torch.empty(xg.beam_select_workspace(xg.XG2_BF16, 1, K, V, n), dtype=torch.uint8, device="cuda")
    xg.beam_select(logits.data_ptr(), xg.XG2_BF16, 1, K, V, stride, d_scores.data_ptr(), n, o[0].data_ptr(), o[1].data_ptr(), o[2].data_ptr(), work.data_ptr(), work.numel(),
                   bitmask_ptr=mask.data_ptr(), bm_row_stride_words=words, eos_id=0, out_finished_ptr=o[3].data_ptr(), stream=_stream())
    want = ref.select(ref.from_bf16(x), allowed, scores, None, 1, K, n, False, 0)
    assert all(np.array_equal(g.cpu().numpy().reshape(1, n), w) for g, w in zip(o[1:], want[1:]))
    assert (np.abs(o[0].cpu().numpy() - want[0][0]) <= ref.score_tolerance(V, want[0][0])).all()


def test_calls_at_the_same_time(xg):
    """Two calls on two streams, each with its own workspace, and the same call again: every result the same."""
    import torch
    rng = np.random.default_rng(15)
    a, b = (Call(xg, *_inputs(rng, 4, 8, 30011, "mixed"), 4, 8, 16, False, "bf16") for _ in range(2))
    wa, wb = a.check(), b.check()
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        with torch.cuda.stream(sa):
            a.run()
        with torch.cuda.stream(sb):
            b.run()
    torch.cuda.synchronize()
    for c, w in ((a, wa), (b, wb)):
        assert all(np.array_equal(p, q) for p, q in zip(c.outputs(), w))


def test_captured_and_replayed(xg):
    import torch
    rng = np.random.default_rng(16)
    x, allowed, scores, finished = _inputs(rng, 3, 5, 20001, "mixed")
    c = Call(xg, x, allowed, scores, finished, 3, 5, 12, True, "f32")
    c.check()
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        c.run()
    for k in range(4):
        scores = np.where(np.isfinite(scores), -rng.random(15) * 4 - 1, scores)
        c.scores = scores.astype(np.float32)
        c.d_scores.copy_(torch.from_numpy(c.scores))
        for t in c.out:
            t[4:-4] = 5
        graph.replay()
        got = c.outputs()
        want = ref.select(c.x, c.allowed, c.scores, finished, 3, 5, 12, True, 0)
        assert all(np.array_equal(g, w) for g, w in zip(got[1:], want[1:])), k
        torch.zeros(1000, device="cuda").sum().item()                # the program's own work between the replays
