"""Timing cases of beam search under a grammar: the operators that choose tokens from masked logits and follow the choice.

A case is a dict of plain values; `prepare` makes what a program has in hand before the call, `run` is one pass.  The paths:

  select     the best candidates of every group of beams: log-probabilities over the tokens that a bitmask allows (or over all
             tokens), added to the beams' scores, the best of all beams and tokens with where they come from
  step       one step of the search: masks of the matcher slots, selection, slots reordered by the chosen parents, the chosen
             tokens accepted
  rows       the beams' rows of an attention cache reordered in place, every group within the positions that its beams differ in
  backtrace  the sequences of all beams from the steps' tokens and parents

Where `own` is false, everything is done with elementary torch operations; the parser of `step` is then a table of the states of a
byte automaton for the same language.  Row numbers are group * beams + beam throughout, -1 stands for no row and no token.
"""
import functools
import math
import random

import numpy as np
import torch

own = False

PERIOD = 32          # steps after which a program's sequences are done and their slots start over
EOS = 0


def listed():
    return [
        # one request's beams inside a JSON document, few tokens allowed: nothing but latency
        dict(name="select_single", path="select", groups=1, beams=4, vocab=32000, dtype="f32", masks="json", over="allowed", n=8),
        # a small batch in free text without a mask, twice as many candidates as beams
        dict(name="select_free", path="select", groups=16, beams=4, vocab=128256, dtype="bf16", masks="none", over="all", n=8),
        # a vocabulary that no vector width divides, an odd number of beams, the model's own probabilities under all kinds of masks
        dict(name="select_odd_vocab", path="select", groups=37, beams=3, vocab=50021, dtype="bf16", masks="mixed", over="all", n=6),
        # wide beams and many candidates
        dict(name="select_wide", path="select", groups=8, beams=32, vocab=151936, dtype="f32", masks="mixed", over="allowed", n=64),
        # the largest batch, every logit counts
        dict(name="select_large", path="select", groups=128, beams=8, vocab=151936, dtype="bf16", masks="free", over="allowed", n=16),
        # one request's step: launches and latency
        dict(name="step_single", path="step", groups=1, beams=4, vocab=32000, dtype="f32"),
        # a serving batch's step
        dict(name="step_batch", path="step", groups=64, beams=8, vocab=128256, dtype="bf16"),
        # one request's cache after a few generated tokens
        dict(name="rows_single", path="rows", groups=1, beams=4, outer=8, pieces=8, positions=512, width=64, type="bf16", prompt=384, generated=48),
        # a layout with all heads of a position together, prompts and answers of all lengths
        dict(name="rows_ragged", path="rows", groups=19, beams=5, outer=6, pieces=1, positions=301, width=520, type="bf16", prompt=200, generated=100),
        # a batch's caches whose beams differ from the first position on
        dict(name="rows_large", path="rows", groups=32, beams=8, outer=8, pieces=8, positions=256, width=64, type="bf16", prompt=0, generated=256),
        # the answer of one request
        dict(name="backtrace_single", path="backtrace", groups=1, beams=4, steps=128),
        # long answers of a batch
        dict(name="backtrace_long", path="backtrace", groups=64, beams=8, steps=1500),
    ]


def _between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    path = rng.choice(("select", "select", "select", "step", "rows", "rows", "backtrace"))
    beams = _between(rng, 1, 32) if path == "select" else _between(rng, 2, 16)
    if path == "select":
        vocab = _between(rng, 2000, 152000) | 1 if rng.random() < 0.4 else 32 * _between(rng, 64, 4748)
        dtype = rng.choice(("bf16", "f32"))
        most = max(1, min(1024, (155 << 20) * (1 if dtype == "bf16" else 0.5) / vocab) / beams)
        return dict(path=path, groups=max(1, int(_between(rng, 1, most))), beams=beams, vocab=vocab, dtype=dtype, masks=rng.choice(("none", "json", "free", "mixed")),
                    over=rng.choice(("allowed", "all")), n=min(128, beams * rng.randint(1, 3)))
    if path == "step":
        vocab = rng.choice((2048, 32000, 50021, 128256))
        return dict(path=path, groups=max(1, _between(rng, 1, 512) // beams), beams=beams, vocab=vocab, dtype=rng.choice(("bf16", "f32")))
    if path == "rows":
        positions, width = _between(rng, 16, 1024), rng.choice((64, 80, 128, 33))
        pieces, kind = rng.choice((1, 2, 8)), rng.choice(("bf16", "f32", "i8"))
        row = pieces * positions * width * {"bf16": 2, "f32": 4, "i8": 1}[kind]
        outer = rng.randint(1, 8)
        groups = max(1, _between(rng, 1, max(1, min(128, (400 << 20) // (row * outer * beams)))))
        prompt = rng.randrange(positions)
        return dict(path=path, groups=groups, beams=beams, outer=outer, pieces=pieces, positions=positions, width=width, type=kind, prompt=prompt, generated=rng.randint(1, positions - prompt))
    return dict(path=path, groups=max(1, _between(rng, 1, 768) // beams), beams=beams, steps=_between(rng, 2, 1500))


def prepare(case, seed):
    return {"select": _prepare_select, "step": _prepare_step, "rows": _prepare_rows, "backtrace": _prepare_backtrace}[case["path"]](case, seed)


def run(s):
    return {"select": _run_select, "step": _run_step, "rows": _run_rows, "backtrace": _run_backtrace}[s["path"]](s)


def exact(case, seed):
    return {"select": _exact_select, "step": _exact_step, "rows": _exact_rows, "backtrace": _exact_backtrace}[case["path"]](case, seed)


def _dtype(name):
    return {"bf16": torch.bfloat16, "f32": torch.float32, "i8": torch.int8}[name]


# ---- selection -----------------------------------------------------------------------------------------------------------------

def _logits(g, rows, vocab, dtype):
    """A model's logits: a broad bulk and, in every row, a few tokens that stand out."""
    x = torch.randn((rows, vocab), generator=g, device="cuda", dtype=torch.float32).mul_(2.0)
    at = torch.randint(0, vocab, (rows, 24), generator=g, device="cuda")
    x.scatter_add_(1, at, torch.rand((rows, 24), generator=g, device="cuda") * 8 + 2)
    return x.to(dtype)


def _pack(allowed):
    """Truth values [rows, V] -> bitmask [rows, ceil(V / 32)] int32."""
    rows, vocab = allowed.shape
    words = (vocab + 31) // 32
    out = torch.empty((rows, words), dtype=torch.int32, device=allowed.device)
    place = (torch.ones(32, dtype=torch.int64, device=allowed.device) << torch.arange(32, device=allowed.device))
    for r in range(0, rows, 64):
        bits = torch.zeros((min(64, rows - r), words * 32), dtype=torch.int64, device=allowed.device)
        bits[:, :vocab] = allowed[r:r + 64]
        packed = (bits.view(-1, words, 32) * place).sum(2)
        out[r:r + 64] = torch.where(packed >= 1 << 31, packed - (1 << 32), packed).to(torch.int32)
    return out


def _unpack(bitmask, vocab):
    place = torch.arange(32, device=bitmask.device, dtype=torch.int32)
    return ((bitmask[:, :, None] >> place) & 1).view(bitmask.shape[0], -1)[:, :vocab] != 0


def _masks(g, rows, vocab, kind):
    """Bitmasks of rows in free text (nearly all is allowed), in a JSON string (three quarters) and between its parts (few tokens)."""
    kinds = torch.randint(0, 3, (rows,), generator=g, device="cuda") if kind == "mixed" else torch.full((rows,), {"free": 0, "json": 2}[kind], device="cuda")
    share = torch.tensor([0.99, 0.75, 0.0], device="cuda")[kinds]
    few = torch.randint(0, vocab, (rows, 48), generator=g, device="cuda")
    count = torch.randint(1, 49, (rows, 1), generator=g, device="cuda")
    few = torch.where(torch.arange(48, device="cuda") < count, few, few[:, :1])
    out = torch.empty((rows, (vocab + 31) // 32), dtype=torch.int32, device="cuda")
    for r in range(0, rows, 64):
        allowed = torch.rand((min(64, rows - r), vocab), generator=g, device="cuda") < share[r:r + 64, None]
        allowed.scatter_(1, few[r:r + 64], True)
        out[r:r + 64] = _pack(allowed)
    return out


def _select_inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    G, K, V = case["groups"], case["beams"], case["vocab"]
    s = dict(path="select", G=G, K=K, V=V, n=case["n"], over=case["over"])
    s["logits"] = _logits(g, G * K, V, _dtype(case["dtype"]))
    s["bitmask"] = None if case["masks"] == "none" else _masks(g, G * K, V, case["masks"])
    s["scores"] = (torch.rand((G, K), generator=g, device="cuda") * -4 - 8).sort(1, descending=True)[0].view(-1).contiguous()
    # a few beams have ended, and a group in eight has just begun: its other beams are no beams yet
    ended = torch.rand(G * K, generator=g, device="cuda") < 0.06
    s["finished"] = ended.to(torch.int32)
    fresh = (torch.rand((G, 1), generator=g, device="cuda") < 0.125) & (torch.arange(K, device="cuda") > 0)
    s["scores"].masked_fill_(fresh.view(-1), -math.inf)
    return s


def _outputs(G, n):
    new = lambda t: torch.empty((G, n), dtype=t, device="cuda")  # noqa: E731
    return dict(out_scores=new(torch.float32), out_parents=new(torch.int32), out_tokens=new(torch.int32), out_finished=new(torch.int32))


def _prepare_select(case, seed):
    s = _select_inputs(case, seed)
    if own:
        import paper_2601_04426_amd as xg
        s.update(_outputs(s["G"], s["n"]), xg=xg, stream=torch.cuda.current_stream().cuda_stream)
        s["workspace"] = torch.empty(xg.beam_select_workspace(_xg_dtype(xg, s["logits"]), s["G"], s["K"], s["V"], s["n"]), dtype=torch.uint8, device="cuda")
    return s


def _xg_dtype(xg, logits):
    return xg.XG2_BF16 if logits.dtype == torch.bfloat16 else xg.XG2_F32


def _own_select(s, finished):
    xg, mask = s["xg"], s["bitmask"]
    xg.beam_select(s["logits"].data_ptr(), _xg_dtype(xg, s["logits"]), s["G"], s["K"], s["V"], s["V"], s["scores"].data_ptr(), s["n"],
                   s["out_scores"].data_ptr(), s["out_parents"].data_ptr(), s["out_tokens"].data_ptr(), s["workspace"].data_ptr(), s["workspace"].numel(),
                   bitmask_ptr=0 if mask is None else mask.data_ptr(), bm_row_stride_words=0 if mask is None else mask.shape[1],
                   over=xg.XG2_OVER_ALLOWED if s["over"] == "allowed" else xg.XG2_OVER_ALL, finished_ptr=finished.data_ptr(), eos_id=EOS,
                   out_finished_ptr=s["out_finished"].data_ptr(), stream=s["stream"])
    return {"scores": s["out_scores"], "parents": s["out_parents"], "tokens": s["out_tokens"], "finished": s["out_finished"]}


def _plain_select(s, bitmask, finished):
    """In 64 bits: what is chosen hangs on values next to each other."""
    G, K, V, n = s["G"], s["K"], s["V"], s["n"]
    x = s["logits"].to(torch.float64)
    allowed = None if bitmask is None else _unpack(bitmask, V)
    counted = x if allowed is None or s["over"] == "all" else x.masked_fill(~allowed, -math.inf)
    top = counted.max(1, keepdim=True)[0]
    total = (counted - top).exp_().sum(1, keepdim=True).log_() + top
    beam = s["scores"].to(torch.float64)[:, None]
    score = x.add_(beam - total) if allowed is None else x.add_(beam - total).masked_fill_(~allowed, -math.inf)
    done = finished != 0
    score.masked_fill_(done[:, None], -math.inf)
    score[:, 0] = torch.where(done, beam[:, 0], score[:, 0])          # an ended beam: itself, once
    score = score.view(G, K * V)
    # one after the other, the first of equals
    best, at = [], []
    for _ in range(n):
        v, i = score.max(1, keepdim=True)
        best.append(v)
        at.append(i)
        score.scatter_(1, i, -math.inf)
    best, at = torch.cat(best, 1), torch.cat(at, 1)
    none = best == -math.inf
    parent = torch.div(at, V, rounding_mode="floor") + torch.arange(G, device="cuda")[:, None] * K
    from_done = done[parent]
    token = torch.where(none | from_done, -1, at % V).to(torch.int32)
    ended = (none | from_done | (token == EOS)).to(torch.int32)
    return {"scores": best.to(torch.float32), "parents": torch.where(none, -1, parent).to(torch.int32), "tokens": token, "finished": ended}


def _run_select(s):
    return _own_select(s, s["finished"]) if own else _plain_select(s, s["bitmask"], s["finished"])


def _exact_choice(x, allowed, scores, done, G, K, n, over):
    """The definition, row by row; x and allowed [rows, V] (allowed may be None)."""
    V = x.shape[1]
    out = {"scores": np.full((G, n), -np.inf), "parents": np.full((G, n), -1), "tokens": np.full((G, n), -1), "finished": np.ones((G, n), dtype=np.int64)}
    for g in range(G):
        found = []
        for r in range(g * K, g * K + K):
            if scores[r] == -np.inf:
                continue
            if done[r]:
                found.append((-float(scores[r]), r, -1))
                continue
            row = x[r].astype(np.float64)
            ids = np.arange(V) if allowed is None else np.flatnonzero(allowed[r])
            if not len(ids):
                continue
            counted = row if over == "all" else row[ids]
            top = counted.max()
            value = row[ids] + (float(scores[r]) - (math.log(np.exp(counted - top).sum()) + top))
            if len(ids) > n:
                least = np.partition(value, len(ids) - n)[len(ids) - n]
                keep = value >= least
                ids, value = ids[keep], value[keep]
            found += [(-v, r, t) for v, t in zip(value.tolist(), ids.tolist())]
        for j, (v, r, t) in enumerate(sorted(found)[:n]):
            out["scores"][g, j], out["parents"][g, j], out["tokens"][g, j], out["finished"][g, j] = -v, r, t, t < 0 or t == EOS
    return out


def _exact_select(case, seed):
    s = _select_inputs(case, seed)
    allowed = None if s["bitmask"] is None else _unpack(s["bitmask"], s["V"]).cpu().numpy()
    return _exact_choice(s["logits"].float().cpu().numpy(), allowed, s["scores"].double().cpu().numpy(), s["finished"].cpu().numpy(), s["G"], s["K"], s["n"], s["over"])


# ---- one step of the search ------------------------------------------------------------------------------------------------------

_EBNF = (r'''root ::= "[" record ("," record)* "]"
record ::= "{\"name\":" text ",\"count\":" number ",\"open\":" flag "}"
text ::= "\"" [a-z ]{0,24} "\""
number ::= "-"? [0-9]{1,9}
flag ::= "true" | "false"
''')


def _automaton():
    """The same language over bytes: table [states, 256] (-1: no way on), start, final states."""
    table = []

    def state():
        table.append([-1] * 256)
        return len(table) - 1

    def chain(at, text, end=None):
        for k, c in enumerate(text):
            to = end if end is not None and k == len(text) - 1 else state()
            table[at][c] = to
            at = to
        return at
    start = state()
    opened = chain(start, b"[")
    at = chain(opened, b'{"name":"')
    after_text = state()
    for k in range(25):
        table[at][ord('"')] = after_text
        if k < 24:
            to = state()
            for c in b" abcdefghijklmnopqrstuvwxyz":
                table[at][c] = to
            at = to
    at = chain(after_text, b',"count":')
    signed, after_number = state(), None
    table[at][ord("-")] = signed
    comma, first = state(), state()
    for c in b"0123456789":
        table[at][c] = table[signed][c] = first
    digit = first
    for k in range(9):
        table[digit][ord(",")] = comma
        if k < 8:
            to = state()
            for c in b"0123456789":
                table[digit][c] = to
            digit = to
    at = chain(comma, b'"open":')
    after_flag = state()
    chain(at, b"true", after_flag)
    chain(at, b"false", after_flag)
    after_record = chain(after_flag, b"}")
    chain(after_record, b",", None)
    again = table[after_record][ord(",")]
    table[again][ord("{")] = table[opened][ord("{")]
    final = chain(after_record, b"]")
    return np.array(table, dtype=np.int16), start, final


@functools.lru_cache(maxsize=2)
def _vocabulary(size):
    """A synthetic tokenizer (token 0 ends a sequence) and, over it, the automaton's next state [states + 1, V]; the last state is that of
    a sequence that has ended."""
    rng = random.Random(size)
    letters = "abcdefghijklmnopqrstuvwxyz"
    seen = {bytes([b]): None for b in range(256)}
    word = lambda lo, hi: "".join(rng.choice(letters) for _ in range(rng.randint(lo, hi)))  # noqa: E731
    for t in ('{"', '":', '":"', '","', '"name', 'name":', '"count":', ',"count":', '"open":', ',"open":', '":true', "true", "false", "true}", "false},", '},{"', '}]', '"},'):
        seen[t.encode()] = None
    while len(seen) < size - 1:
        u = rng.random()
        if u < 0.6:
            t = (" " if rng.random() < 0.5 else "") + word(1, 7)
        elif u < 0.7:
            t = str(rng.randrange(10 ** rng.randint(1, 5)))
        elif u < 0.8:
            t = word(0, 4) + '",' + rng.choice(('"', '"count', '"count":'))
        else:
            t = "".join(chr(rng.randint(32, 126)) for _ in range(rng.randint(1, 8)))
        seen[t.encode()] = None
    tokens = [b""] + list(seen)
    table, start, final = _automaton()
    n = len(table)
    ways = np.vstack([table, np.full((1, 256), -1, dtype=np.int16)])   # (the last row: where -1 leads)
    longest = max(map(len, tokens))
    text = np.zeros((size, longest), dtype=np.uint8)
    length = np.array([len(t) for t in tokens])
    for i, t in enumerate(tokens):
        text[i, :len(t)] = np.frombuffer(t, dtype=np.uint8)
    state = np.repeat(np.arange(n, dtype=np.int16)[:, None], size, 1)
    for k in range(longest):
        state = np.where(length > k, ways[state, text[:, k]], state)
    state[:, EOS] = -1
    state[final, EOS] = n
    state = np.vstack([state, np.full((1, size), -1, dtype=np.int16)])
    state[n, EOS] = n                                                  # a sequence that has ended may only end
    ends = np.flatnonzero([b"]" in t for t in tokens])
    return tokens, torch.from_numpy(state.astype(np.int64)), start, torch.from_numpy(ends)


def _step_inputs(case, seed):
    G, K, V = case["groups"], case["beams"], case["vocab"]
    tokens, table, start, ends = _vocabulary(V)
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(path="step", G=G, K=K, V=V, n=K, over="allowed", turn=0, start=start)
    s["logits"] = _logits(g, G * K, V, torch.float32)
    s["logits"][:, ends.cuda()] -= 12                                  # long lists
    s["logits"] = s["logits"].to(_dtype(case["dtype"]))
    s["scores"] = (torch.rand((G, K), generator=g, device="cuda") * -2 - 8).sort(1, descending=True)[0].view(-1).contiguous()
    # where the beams are: random tokens of the language, up to 24 of them, none that closes the list
    rng = np.random.default_rng(seed)
    way = table.numpy().copy()
    way[:, ends.numpy()] = -1
    choices = [np.flatnonzero(row >= 0) for row in way]
    at = np.full(G * K, start)
    depth = rng.integers(0, 25, G * K)
    lead = np.full((int(depth.max()), G * K), -1, dtype=np.int32)
    for k in range(len(lead)):
        for b in np.flatnonzero(depth > k):
            lead[k, b] = rng.choice(choices[at[b]])
            at[b] = way[at[b], lead[k, b]]
    s["state"] = torch.from_numpy(at).cuda()
    s["finished"] = torch.zeros(G * K, dtype=torch.int32, device="cuda")
    return s, tokens, table, lead


def _prepare_step(case, seed):
    s, tokens, table, lead = _step_inputs(case, seed)
    R, V = s["G"] * s["K"], s["V"]
    s["fresh"] = torch.full((R,), -2, dtype=torch.int32, device="cuda")
    if own:
        import paper_2601_04426_amd as xg
        stream = torch.cuda.current_stream().cuda_stream
        vocab = _handle(V)
        cache = xg.compile_grammar(vocab, _EBNF, stream=stream)
        slots = xg.DeviceBatch(vocab, R)
        slots.assign(cache, stream=stream)
        s.update(_outputs(s["G"], s["n"]), xg=xg, stream=stream, slots=slots, W=vocab.words)
        s["bitmask"] = torch.zeros((R, vocab.words), dtype=torch.int32, device="cuda")
        s["status"] = torch.zeros(R, dtype=torch.int32, device="cuda")
        s["workspace"] = torch.empty(xg.beam_select_workspace(_xg_dtype(xg, s["logits"]), s["G"], s["K"], V, s["n"]), dtype=torch.uint8, device="cuda")
        for row in torch.from_numpy(lead).cuda().unbind(0):
            slots.accept_tokens(row.data_ptr(), s["status"].data_ptr(), stream)
    else:
        s["table"], s["masks"] = table.cuda(), _pack((table >= 0).cuda())
    return s


@functools.lru_cache(maxsize=2)
def _handle(size):
    import paper_2601_04426_amd as xg
    return xg.Vocab(_vocabulary(size)[0], EOS, [EOS])


def _run_step(s):
    fresh = s["turn"] == PERIOD - 1                                    # the sequences' last step: their slots are given to new ones
    s["turn"] = (s["turn"] + 1) % PERIOD
    if own:
        s["slots"].fill_next_token_bitmask(s["bitmask"].data_ptr(), s["W"], s["stream"])
        out = _own_select(s, s["finished"])
        s["slots"].reorder(s["K"], s["out_parents"].data_ptr(), 0, s["stream"])
        s["slots"].accept_tokens((s["fresh"] if fresh else s["out_tokens"]).data_ptr(), s["status"].data_ptr(), s["stream"])
        s["finished"].copy_(s["out_finished"].view(-1))
        out.update(bitmask=s["bitmask"], status=s["status"])
    else:
        mask = s["masks"][s["state"]]
        out = _plain_select(s, mask, s["finished"])
        parent, token = out["parents"].view(-1).to(torch.int64), out["tokens"].view(-1).to(torch.int64)
        state = torch.where(parent >= 0, s["state"][parent.clamp(min=0)], s["state"])
        to = s["table"][state, token.clamp(min=0)]
        s["state"] = torch.full_like(state, s["start"]) if fresh else torch.where((token >= 0) & (to >= 0), to, state)
        s["finished"] = out["finished"].view(-1).clone()
        out.update(bitmask=mask, status=torch.zeros_like(s["finished"]) if fresh else torch.where((token >= 0) & (to < 0), -3, 0).to(torch.int32))
    if fresh:
        s["finished"].zero_()
    return out


def _exact_step(case, seed):
    s, _, table, _ = _step_inputs(case, seed)
    table, state = table.numpy(), s["state"].cpu().numpy()
    allowed = table[state] >= 0
    out = _exact_choice(s["logits"].float().cpu().numpy(), allowed, s["scores"].double().cpu().numpy(), s["finished"].cpu().numpy(), s["G"], s["K"], s["n"], s["over"])
    W = (s["V"] + 31) // 32
    bits = np.zeros((len(state), W * 32), dtype=np.uint8)
    bits[:, :s["V"]] = allowed
    out["bitmask"] = np.packbits(bits, axis=1, bitorder="little").view("<i4").astype(np.int64)
    out["status"] = np.zeros(len(state), dtype=np.int64)
    return out


# ---- rows of a cache -------------------------------------------------------------------------------------------------------------

def _rows_inputs(case, seed):
    G, K = case["groups"], case["beams"]
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(path="rows", G=G, K=K, turn=0)
    shape = (case["outer"], G * K, case["pieces"], case["positions"], case["width"])
    kind = _dtype(case["type"])
    if kind == torch.int8:
        s["data"] = torch.randint(-128, 128, shape, generator=g, device="cuda", dtype=torch.int8)
    else:
        s["data"] = torch.randn(shape, generator=g, device="cuda", dtype=kind)
    # what a selection chooses: the better beams more than once, most beams in their own place or another's
    parents = (torch.rand((8, G, K), generator=g, device="cuda") ** 1.7 * K).to(torch.int32).clamp_(max=K - 1).sort(2)[0]
    s["parents"] = list((parents + torch.arange(G, device="cuda", dtype=torch.int32)[:, None] * K).view(8, -1).contiguous().unbind(0))
    # a group's beams have their prompt in common
    begin = torch.randint(case["prompt"] // 2, case["prompt"] + 1, (G,), generator=g, device="cuda", dtype=torch.int32)
    length = torch.randint(case["generated"] // 2 + 1, case["generated"] + 1, (G,), generator=g, device="cuda", dtype=torch.int32)
    s["begin"], s["end"] = begin, begin + length
    return s


def _prepare_rows(case, seed):
    s = _rows_inputs(case, seed)
    if own:
        import paper_2601_04426_amd as xg
        s.update(xg=xg, stream=torch.cuda.current_stream().cuda_stream)
    return s


def _run_rows(s):
    data, parents = s["data"], s["parents"][s["turn"]]
    s["turn"] = (s["turn"] + 1) % len(s["parents"])
    if own:
        size = data.element_size()
        s["xg"].beam_reorder_rows(data.data_ptr(), s["G"], s["K"], parents.data_ptr(), row_stride=data.stride(1) * size, outer=data.shape[0], outer_stride=data.stride(0) * size,
                                  pieces=data.shape[2], piece_stride=data.stride(2) * size, positions=data.shape[3], position_bytes=data.stride(3) * size,
                                  begin_ptr=s["begin"].data_ptr(), end_ptr=s["end"].data_ptr(), stream=s["stream"])
        return data
    at = torch.arange(data.shape[3], device="cuda")
    inside = (at >= s["begin"].repeat_interleave(s["K"], output_size=data.shape[1])[:, None]) & (at < s["end"].repeat_interleave(s["K"], output_size=data.shape[1])[:, None])
    data.copy_(torch.where(inside[None, :, None, :, None], data[:, parents.to(torch.int64)], data))
    return data


def _exact_rows(case, seed):
    s = _rows_inputs(case, seed)
    if s["data"].numel() > 1 << 28:
        return None
    data = s["data"].float().cpu().numpy().astype(np.int64 if case["type"] == "i8" else np.float64)
    parents, begin, end = s["parents"][0].cpu().numpy(), s["begin"].cpu().numpy(), s["end"].cpu().numpy()
    out = data.copy()
    for r, p in enumerate(parents):
        g = r // s["K"]
        out[:, r, :, begin[g]:end[g]] = data[:, p, :, begin[g]:end[g]]
    return out


# ---- the sequences ---------------------------------------------------------------------------------------------------------------

def _prepare_backtrace(case, seed):
    G, K, T = case["groups"], case["beams"], case["steps"]
    rng = np.random.default_rng(seed)
    beam = np.sort((rng.random((T, G, K)) ** 1.7 * K).astype(np.int32), 2)
    # a beam that ends stays where it is: the last place of its group, from a step of its own on
    last = rng.integers(1, 2 * T, G)
    ended = np.arange(T)[:, None] >= last
    beam[:, :, K - 1] = np.where(ended, K - 1, beam[:, :, K - 1])
    tokens = rng.integers(1, 100000, (T, G, K)).astype(np.int32)
    tokens[:, :, K - 1] = np.where(ended, np.where(np.arange(T)[:, None] == last, EOS, -1), tokens[:, :, K - 1])
    parents = beam + (np.arange(G, dtype=np.int32) * K)[:, None]
    s = dict(path="backtrace", G=G, K=K, T=T, tokens=torch.from_numpy(tokens.reshape(T, G * K)).cuda(), parents=torch.from_numpy(parents.reshape(T, G * K).astype(np.int32)).cuda())
    if own:
        import paper_2601_04426_amd as xg
        s.update(xg=xg, stream=torch.cuda.current_stream().cuda_stream, out=torch.empty((G * K, T), dtype=torch.int32, device="cuda"),
                 lengths=torch.empty(G * K, dtype=torch.int32, device="cuda"))
    return s


def _run_backtrace(s):
    T, R = s["T"], s["G"] * s["K"]
    if own:
        s["xg"].beam_backtrace(s["tokens"].data_ptr(), s["parents"].data_ptr(), T, R, s["G"], s["K"], s["out"].data_ptr(), T, lengths_ptr=s["lengths"].data_ptr(), stream=s["stream"])
        return {"tokens": s["out"], "lengths": s["lengths"]}
    row = torch.arange(R, device="cuda")
    out = torch.empty((T, R), dtype=torch.int32, device="cuda")
    for t in range(T - 1, -1, -1):
        out[t] = s["tokens"][t][row]
        row = s["parents"][t][row]
    out = out.t().contiguous()
    return {"tokens": out, "lengths": torch.where(out >= 0, torch.arange(1, T + 1, device="cuda"), 0).max(1)[0].to(torch.int32)}


def _exact_backtrace(case, seed):
    s = _prepare_backtrace(case, seed)
    tokens, parents = s["tokens"].cpu().numpy(), s["parents"].cpu().numpy()
    T, R = tokens.shape
    out, length = np.empty((R, T), dtype=np.int64), np.zeros(R, dtype=np.int64)
    for r in range(R):
        at = r
        for t in range(T - 1, -1, -1):
            out[r, t] = tokens[t, at]
            if out[r, t] >= 0 and length[r] == 0:
                length[r] = t + 1
            at = parents[t, at]
    return {"tokens": out, "lengths": length}


# ----------------------------------------------------------------------------------------------------------------------------------

def work(case):
    """Bytes: logits that count once (between the parts of a JSON document, where some two dozen tokens a row are allowed and the
    softmax goes over them, those alone), masks once, the moved rows read and written once (about two in three of a group's), tokens and
    parents once.  Operations: an exponential, a product, two sums and a comparison for every logit that counts."""
    path, rows = case["path"], case["groups"] * case["beams"]
    if path in ("select", "step"):
        V, size = case["vocab"], 2 if case["dtype"] == "bf16" else 4
        masks, over = case.get("masks", "step"), case.get("over", "allowed")
        count = {"none": V, "free": V, "json": 24, "mixed": 0.58 * V, "step": 0.2 * V}[masks] if over == "allowed" else V
        mask = 0 if masks == "none" else rows * ((V + 31) // 32) * 4
        return {"bytes": int(rows * count * size) + mask * (2 if path == "step" else 1) + 16 * case["groups"] * case.get("n", case["beams"]), "flops": int(5 * rows * count)}
    if path == "rows":
        length = 0.75 * case["generated"]
        return {"bytes": int(2 * 0.66 * rows * case["outer"] * case["pieces"] * length * case["width"] * {"bf16": 2, "f32": 4, "i8": 1}[case["type"]]), "flops": 0}
    return {"bytes": rows * case["steps"] * 12, "flops": 0}
