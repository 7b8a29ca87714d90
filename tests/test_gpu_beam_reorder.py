"""Reordering of matcher slots and of a buffer's rows by parents, and the sequences of the beams.  Bit for bit."""
import random

import numpy as np
import pytest

import beam_reference as ref
import gen
import oracle
from helpers import load

pytestmark = pytest.mark.gpu

OK, EINVAL, EOVERFLOW = 0, -1, -4


@pytest.fixture(scope="module")
def xg():
    import torch
    assert torch.cuda.is_available()
    import paper_2601_04426_amd as xg
    return xg


def _stream():
    import torch
    return torch.cuda.current_stream().cuda_stream


def _parents(rng, G, K, stray=0.0):
    """Random parents of the same group; some rows keep their place by -1, and a share of strays names other rows or none."""
    p = rng.integers(0, K, (G, K)) + np.arange(G)[:, None] * K
    p = np.where(rng.random((G, K)) < 0.15, -1, p)
    if stray:
        wild = rng.choice([-2, -7, G * K, G * K + 5, 2 ** 31 - 1, -2 ** 31] + list(range(G * K)), (G, K))
        p = np.where(rng.random((G, K)) < stray, wild, p)
    return p.reshape(-1).astype(np.int32)


# ---- matcher slots ---------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("G,K", [(1, 1), (1, 2), (3, 4), (2, 16), (1, 17), (2, 33), (1, 64), (7, 5)])
def test_slots_follow_their_parents(xg, G, K):
    """Slots of three grammars, one per group in turn: random allowed tokens, reorderings with parents taken up several times; every
    mask equals the oracle's for the history that the slot has by then, ended sequences and untouched slots among them."""
    import torch
    cfg, vocab, va = load(1)
    grammars = [cfg.grammars[0], ('root ::= "[" ws (num (ws "," ws num)*)? ws "]"\nnum ::= "-"? [0-9]{1,4}\nws ::= [ \t\n]*\n', "root"),
                ('root ::= item+\nitem ::= "<" [a-z]{1,8} ">" | [A-Z ]\n', "root")]
    caches = [xg.compile_grammar(vocab, e, r, stream=_stream()) for e, r in grammars]
    orcs = [oracle.Oracle(e, r) for e, r in grammars]
    rng, pick = np.random.default_rng(G * 100 + K), random.Random(G * 100 + K)
    B = G * K
    db = xg.DeviceBatch(vocab, B)
    for b in range(B):
        db.assign(caches[b // K % 3], rows=[b], stream=_stream())
    ids, status, moved = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(3))
    bitmask = torch.zeros((B, vocab.words), dtype=torch.int32, device="cuda")
    state = [(b // K % 3, b"", False) for b in range(B)]             # grammar, history, ended
    memo = {}

    def mask(s):
        if s not in memo:
            want = orcs[s[0]].mask(s[1], va)
            if s[2]:
                want = np.zeros(vocab.size, dtype=bool)
                want[cfg.vocab.eos_id] = True
            memo[s] = want
        return memo[s]
    for step in range(10):
        parents = _parents(rng, G, K, stray=0.2 if step % 3 == 2 else 0.0)
        p = torch.from_numpy(parents).cuda()
        db.reorder(K, p.data_ptr(), moved.data_ptr(), _stream())
        inside = (parents == -1) | ((parents >= np.arange(B) // K * K) & (parents < np.arange(B) // K * K + K))
        assert np.array_equal(moved.cpu().numpy(), np.where(inside, OK, EINVAL)), step
        state = ref.reorder(state, parents, G, K)
        db.fill_next_token_bitmask(bitmask.data_ptr(), vocab.words, _stream())
        got = bitmask.cpu().numpy()
        nxt = np.full(B, -1, dtype=np.int32)
        for b, s in enumerate(state):
            want = mask(s)
            assert np.array_equal(got[b], oracle.pack_bitmask(want)), (step, b, s)
            if not s[2] and pick.random() < 0.8:
                nxt[b] = pick.choice(np.flatnonzero(want).tolist())
        ids.copy_(torch.from_numpy(nxt))
        db.accept_tokens(ids.data_ptr(), status.data_ptr(), _stream())
        assert not status.cpu().numpy().any()
        for b, t in enumerate(nxt):
            if t == cfg.vocab.eos_id:
                state[b] = (state[b][0], state[b][1], True)
            elif t > 0:
                state[b] = (state[b][0], state[b][1] + cfg.vocab.tokens[t], False)


def test_slots_with_deep_contexts_and_errors(xg):
    """A right-recursive rule makes every token add a set of items: contexts up to a slot's capacity are taken over whole, and a slot
    that has exceeded it hands on its error until it is reset."""
    import torch
    toks = [b"", b"x", b"y", b"xx"]
    vocab = xg.Vocab(toks, 0, [0])
    va = oracle.VocabArrays(toks, 0, [0])
    ebnf = 'root ::= a\na ::= "x" a | "y"\n'
    cache = xg.compile_grammar(vocab, ebnf, "root", stream=_stream())
    orc = oracle.Oracle(ebnf, "root")
    K = 4
    db = xg.DeviceBatch(vocab, K)
    db.assign(cache, stream=_stream())
    status = torch.zeros(K, dtype=torch.int32, device="cuda")
    bm = torch.zeros((K, 1), dtype=torch.int32, device="cuda")

    def put(v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")
    n = [0] * K                                                      # every slot's x's
    for step in range(230):
        db.accept_tokens(put([1, 3 if step < 100 else -1, -1, 1 if step < 70 else -1]).data_ptr(), status.data_ptr(), _stream())
        assert not status.cpu().numpy().any()
        n = [n[0] + 1, n[1] + 2 * (step < 100), n[2], n[3] + (step < 70)]
        if step % 23 == 22:
            parents = [0, 1, 0 if step % 2 else 1, 3]
            db.reorder(K, put(parents).data_ptr(), 0, _stream())
            n = [n[p] for p in parents]
            db.fill_next_token_bitmask(bm.data_ptr(), 1, _stream())
            got = bm.cpu().numpy()
            assert all(np.array_equal(got[b], oracle.pack_bitmask(orc.mask(b"x" * n[b], va))) for b in range(K)), step
            assert [db.row_info(b)["sets"] for b in range(K)] == [db.row_info(p)["sets"] for p in parents]
    for _ in range(30):
        db.accept_tokens(put([1, -1, -1, -1]).data_ptr(), status.data_ptr(), _stream())
    assert status.cpu().numpy()[0] == EOVERFLOW
    db.reorder(K, put([1, 0, 0, 3]).data_ptr(), status.data_ptr(), _stream())
    assert not status.cpu().numpy().any()
    assert [db.row_info(b)["error"] for b in range(K)] == [0, 1, 1, 0]
    db.accept_tokens(put([1, 1, -2, 1]).data_ptr(), status.data_ptr(), _stream())
    assert status.cpu().numpy().tolist() == [OK, EOVERFLOW, OK, OK]
    db.fill_next_token_bitmask(bm.data_ptr(), 1, _stream())
    got = bm.cpu().numpy()
    for b, x in ((0, n[1] + 1), (2, 0), (3, n[3] + 1)):
        assert np.array_equal(got[b], oracle.pack_bitmask(orc.mask(b"x" * x, va))), b


def test_slots_of_different_grammars_in_a_group(xg):
    """A slot takes over its parent's grammar with its state, and keeps it; a slot that is reset meanwhile starts again with another."""
    import torch
    cfg, vocab, va = load(1)
    grammars = [cfg.grammars[0], ('root ::= "[" ws (num (ws "," ws num)*)? ws "]"\nnum ::= "-"? [0-9]{1,4}\nws ::= [ \t\n]*\n', "root"),
                ('root ::= item+\nitem ::= "<" [a-z]{1,8} ">" | [A-Z ]\n', "root")]
    caches = [xg.compile_grammar(vocab, e, r, stream=_stream()) for e, r in grammars]
    orcs = [oracle.Oracle(e, r) for e, r in grammars]
    G, K = 3, 7
    B = G * K
    rng, pick = np.random.default_rng(5), random.Random(5)
    db = xg.DeviceBatch(vocab, B)
    state = [(b % 3, b"") for b in range(B)]
    for b in range(B):
        db.assign(caches[b % 3], rows=[b], stream=_stream())
    status = torch.zeros(B, dtype=torch.int32, device="cuda")
    bitmask = torch.zeros((B, vocab.words), dtype=torch.int32, device="cuda")
    for step in range(8):
        parents = _parents(rng, G, K)
        p = torch.from_numpy(parents).cuda()
        db.reorder(K, p.data_ptr(), p.data_ptr(), _stream())         # (the statuses may take the parents' place)
        assert not p.cpu().numpy().any()
        state = ref.reorder(state, parents, G, K)
        if step == 4:
            for b in (0, 8, 20):
                db.assign(caches[(b + 1) % 3], rows=[b], stream=_stream())
                state[b] = ((b + 1) % 3, b"")
        db.fill_next_token_bitmask(bitmask.data_ptr(), vocab.words, _stream())
        got = bitmask.cpu().numpy()
        nxt = np.full(B, -1, dtype=np.int32)
        for b, (c, h) in enumerate(state):
            want = orcs[c].mask(h, va)
            assert np.array_equal(got[b], oracle.pack_bitmask(want)), (step, b)
            can = [t for t in np.flatnonzero(want).tolist() if t != cfg.vocab.eos_id]
            if can and pick.random() < 0.9:
                nxt[b] = pick.choice(can)
                state[b] = (c, h + cfg.vocab.tokens[nxt[b]])
        ids = torch.from_numpy(nxt).cuda()
        db.accept_tokens(ids.data_ptr(), status.data_ptr(), _stream())
        assert not status.cpu().numpy().any()


def test_slots_refusals(xg):
    import torch
    cfg, vocab, _ = load(1)
    db = xg.DeviceBatch(vocab, 6)
    p = torch.arange(6, dtype=torch.int32, device="cuda")
    with pytest.raises(xg.Xg2Error) as e:                            # slots without a cache
        db.reorder(3, p.data_ptr(), 0, _stream())
    assert e.value.code == EINVAL
    db.assign(xg.compile_grammar(vocab, *cfg.grammars[0], stream=_stream()), stream=_stream())
    for beams, ptr, st in ((0, p.data_ptr(), 0), (65, p.data_ptr(), 0), (4, p.data_ptr(), 0), (3, 0, 0), (3, p.data_ptr() + 2, 0), (3, p.data_ptr(), p.data_ptr() + 1)):
        with pytest.raises(xg.Xg2Error) as e:
            db.reorder(beams, ptr, st, _stream())
        assert e.value.code == EINVAL, (beams, ptr, st)
    db.reorder(3, p.data_ptr(), 0, _stream())


# ---- rows of a buffer ------------------------------------------------------------------------------------------------

def _rows_case(xg, rng, G, K, outer, pieces, positions, width, layout, windows, shift):
    """A buffer of bytes with a guard around it, in one of the layouts that the header names."""
    import torch
    R = G * K
    shape = {"heads": (outer, R, pieces, positions, width), "rows first": (R, outer, pieces, positions, width), "rows inside": (outer, pieces, R, positions, width)}[layout]
    n = int(np.prod(shape))
    raw = rng.integers(0, 256, n + 128, dtype=np.uint8)
    d = torch.from_numpy(raw).cuda()
    base = 64 + shift
    want = raw.copy()
    view = want[base:base + n].reshape(shape)
    canon = {"heads": view, "rows first": view.transpose(1, 0, 2, 3, 4), "rows inside": view.transpose(0, 2, 1, 3, 4)}[layout]
    P = positions * width
    strides = {"heads": dict(row_stride=pieces * P, outer=outer, outer_stride=R * pieces * P, pieces=pieces, piece_stride=P),
               "rows first": dict(row_stride=outer * pieces * P, outer=1, outer_stride=0, pieces=outer * pieces, piece_stride=P),
               "rows inside": dict(row_stride=P, outer=outer, outer_stride=pieces * R * P, pieces=pieces, piece_stride=R * P)}[layout]
    parents = _parents(rng, G, K, stray=0.1)
    begin = rng.integers(-2, positions + 2, G).astype(np.int32)
    end = rng.integers(-2, positions + 3, G).astype(np.int32)
    if windows == "none":
        begin, end = np.zeros(G, dtype=np.int32), np.full(G, positions, dtype=np.int32)
    elif windows == "begin":
        end = np.full(G, positions, dtype=np.int32)
    elif windows == "end":
        begin = np.zeros(G, dtype=np.int32)
    before = canon.copy()
    for r in range(R):
        p, g = int(parents[r]), r // K
        lo, hi = max(0, begin[g]), min(positions, end[g])
        if g * K <= p < g * K + K and lo < hi:
            canon[:, r, :, lo:hi] = before[:, p, :, lo:hi]
    dp, db, de = (torch.from_numpy(a).cuda() for a in (parents, begin, end))
    xg.beam_reorder_rows(d.data_ptr() + base, G, K, dp.data_ptr(), positions=positions, position_bytes=width, begin_ptr=db.data_ptr() if windows in ("both", "begin") else 0,
                         end_ptr=de.data_ptr() if windows in ("both", "end") else 0, stream=_stream(), **strides)
    got = d.cpu().numpy()
    assert np.array_equal(got, want), (G, K, outer, pieces, positions, width, layout, windows, shift, np.flatnonzero(got != want)[:4])


@pytest.mark.parametrize("K", [1, 2, 4, 5, 8, 9, 16, 17, 32, 33, 64])
def test_rows_of_all_sizes(xg, K):
    rng = np.random.default_rng(K)
    for k, (positions, width) in enumerate([(1, 1), (3, 5), (1, 16), (7, 16), (33, 66), (130, 128), (600, 30), (17, 1040)]):
        for layout in ("heads", "rows first", "rows inside"):
            _rows_case(xg, rng, 1 + (k + K) % 3, K, 1 + k % 2, 1 + (k + 1) % 3, positions, width, layout, ("both", "none", "begin", "end")[k % 4], (0, 1, 2, 4, 8, 3)[(k + K) % 6])


def test_rows_permutations_and_cycles(xg):
    """Every row moves: cycles, one parent for all, a shift; twice in a row."""
    import torch
    for K in (3, 8, 20, 64):
        for name, p in (("cycle", np.roll(np.arange(K), 1)), ("all one", np.full(K, K - 1)), ("shift", np.maximum(np.arange(K) - 1, 0)), ("reverse", np.arange(K)[::-1])):
            x = torch.randn((2, K, 3, 40, 24), device="cuda")
            d, q = x.clone(), torch.from_numpy(p.astype(np.int32).copy()).cuda()
            for _ in range(2):
                xg.beam_reorder_rows(d.data_ptr(), 1, K, q.data_ptr(), row_stride=3 * 40 * 96, positions=40, position_bytes=96, outer=2, outer_stride=K * 3 * 40 * 96, pieces=3,
                                     piece_stride=40 * 96, stream=_stream())
                x = x[:, q.long()]
            assert torch.equal(d, x), (K, name)


@pytest.mark.parametrize("K", [2, 3, 11, 24, 64])
def test_rows_past_the_caches(xg, K):
    """Buffers beyond 256 MB, pieces whose begins and ends lie anywhere."""
    import torch
    positions, width, pieces = 1003, 135, 3
    G = (300 << 20) // (K * pieces * positions * width) + 1
    g = torch.Generator(device="cuda").manual_seed(K)
    d = torch.randint(0, 256, (G * K, pieces, positions, width), generator=g, device="cuda", dtype=torch.uint8)
    p = torch.randint(0, K, (G, K), generator=g, device="cuda", dtype=torch.int32) + torch.arange(G, device="cuda", dtype=torch.int32)[:, None] * K
    begin = torch.randint(0, positions, (G,), generator=g, device="cuda", dtype=torch.int32)
    want = d[p.view(-1).long()]
    t = torch.arange(positions, device="cuda")
    outside = (t[None, :] < begin[:, None]).repeat_interleave(K, 0)
    want = torch.where(outside[:, None, :, None], d, want)
    xg.beam_reorder_rows(d.data_ptr(), G, K, p.data_ptr(), row_stride=pieces * positions * width, positions=positions, position_bytes=width, pieces=pieces,
                         piece_stride=positions * width, begin_ptr=begin.data_ptr(), stream=_stream())
    assert torch.equal(d, want)


def test_rows_of_many_groups_and_pieces(xg):
    """More groups than one dimension of a grid takes; rows of very many small pieces; one long piece."""
    rng = np.random.default_rng(31)
    _rows_case(xg, rng, 33003, 2, 1, 2, 3, 5, "heads", "both", 0)
    _rows_case(xg, rng, 2, 3, 3, 200_003, 2, 3, "heads", "both", 1)
    _rows_case(xg, rng, 1, 5, 1, 1, 1_000_003, 7, "heads", "both", 3)
    _rows_case(xg, rng, 1, 40, 1, 1, 100_003, 7, "heads", "none", 2)


def test_rows_beyond_4_gib(xg):
    """Offsets beyond 32 bits: rows of 600 MB, and a buffer whose outer parts lie 5 GiB apart."""
    import torch
    K, size = 8, 600 << 20
    d = torch.empty(K * size, dtype=torch.uint8, device="cuda")
    for k in range(K):
        d[k * size:(k + 1) * size] = k + 1
    p = torch.tensor([7, 1, 2, 0, 4, 5, 6, 3], dtype=torch.int32, device="cuda")
    begin, end = (torch.tensor([v], dtype=torch.int32, device="cuda") for v in (599, 600))
    xg.beam_reorder_rows(d.data_ptr(), 1, K, p.data_ptr(), row_stride=size, positions=600, position_bytes=1 << 20, begin_ptr=begin.data_ptr(), end_ptr=end.data_ptr(), stream=_stream())
    for k, q in enumerate(p.tolist()):
        assert (d[(k + 1) * size - (1 << 20):(k + 1) * size] == q + 1).all() and (d[k * size:(k + 1) * size - (1 << 20)] == k + 1).all(), k
    xg.beam_reorder_rows(d.data_ptr(), 1, 2, p.data_ptr() + 4, row_stride=4096, positions=1, position_bytes=4096, outer=2, outer_stride=(K - 1) * size, stream=_stream())   # parents 1, 2: row 0 takes row 1
    assert (d[:4096] == 1).all()
    d[:4096], d[4096:8192] = 100, 101
    d[(K - 1) * size:(K - 1) * size + 4096], d[(K - 1) * size + 4096:(K - 1) * size + 8192] = 102, 103
    xg.beam_reorder_rows(d.data_ptr(), 1, 2, torch.tensor([1, 0], dtype=torch.int32, device="cuda").data_ptr(), row_stride=4096, positions=1, position_bytes=4096, outer=2,
                         outer_stride=(K - 1) * size, stream=_stream())
    assert [int(d[o]) for o in (0, 4095, 4096, 8191, 8192)] == [101, 101, 100, 100, 1]
    assert [int(d[(K - 1) * size + o]) for o in (0, 4095, 4096, 8191)] == [103, 103, 102, 102]


# ---- sequences -------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("G,K", [(1, 1), (3, 2), (2, 5), (1, 16), (2, 33), (1, 64), (300, 3)])
def test_sequences(xg, G, K):
    import torch
    rng = np.random.default_rng(G + K)
    R = G * K
    for T, stray, pad, stride in ((1, 0.0, 0, 0), (2, 0.0, 3, 1), (15, 0.02, 0, 0), (16, 0.0, 0, 5), (17, 0.0, 1, 0), (63, 0.01, 2, 0), (64, 0.0, 0, 0), (65, 0.0, 0, 2), (257, 0.002, 0, 3), (1025, 0.0, 7, 0)):
        tokens = rng.integers(-1, 1000, (T, R + stride)).astype(np.int32)
        parents = np.full((T, R + stride), 12345, dtype=np.int32)
        for t in range(T):
            parents[t, :R] = rng.integers(0, K, R) + np.arange(R) // K * K
        wild = rng.random((T, R)) < stray
        parents[:, :R][wild] = rng.choice(np.array([-1, -5, R, 2 ** 31 - 1], dtype=np.int32), wild.sum())
        dt, dp = torch.from_numpy(tokens).cuda(), torch.from_numpy(parents).cuda()
        out = torch.full((R, T + pad), 55, dtype=torch.int32, device="cuda")
        length = torch.full((R + 2,), 55, dtype=torch.int32, device="cuda")
        xg.beam_backtrace(dt.data_ptr(), dp.data_ptr(), T, R + stride, G, K, out.data_ptr(), T + pad, lengths_ptr=length.data_ptr() + 4, stream=_stream())
        want, n = ref.backtrace(tokens[:, :R], parents[:, :R], G, K)
        got = out.cpu().numpy()
        assert np.array_equal(got[:, :T], want), (T, stray)
        assert (got[:, T:] == 55).all() and length[0] == 55 and length[-1] == 55
        assert np.array_equal(length[1:-1].cpu().numpy(), n), T
        out.fill_(3)
        xg.beam_backtrace(dt.data_ptr(), dp.data_ptr(), T, R + stride, G, K, out.data_ptr(), T + pad, stream=_stream())
        assert np.array_equal(out.cpu().numpy()[:, :T], want)


def test_sequences_of_no_steps(xg):
    import torch
    length = torch.full((6,), 9, dtype=torch.int32, device="cuda")
    xg.beam_backtrace(0, 0, 0, 0, 2, 3, 0, 0, lengths_ptr=length.data_ptr(), stream=_stream())
    assert not length.cpu().numpy().any()
