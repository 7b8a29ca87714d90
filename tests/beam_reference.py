"""The operators of beam search by their definitions, in 64 bits on the CPU."""
import math

import numpy as np


def to_bf16(x: np.ndarray) -> np.ndarray:
    """float32 -> the bits of the nearest bfloat16 (ties to even; NaN stays NaN)."""
    u = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    out = ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)
    return np.where(np.isnan(x), np.uint16(0x7FC0), out)


def from_bf16(bits: np.ndarray) -> np.ndarray:
    return (bits.astype(np.uint32) << 16).view(np.float32)


def log_total(row, counted):
    """(log of the sum of exp over the counted tokens, whether infinite logits are among them), NaN and -infinity left out."""
    v = row[counted]
    v = v[~np.isnan(v) & (v != -np.inf)].astype(np.float64)
    if not len(v):
        return -math.inf, False
    if np.isposinf(v).any():
        return math.log(np.isposinf(v).sum()), True
    top = v.max()
    return math.log(math.fsum(np.exp(v - top))) + top, False


def select(logits, allowed, scores, finished, G, K, n, over_all, eos):
    """logits [G * K, V] float32 (NaN and infinities as they come), allowed the same shape or None.  -> scores (64 bits), parents,
    tokens, finished, [G, n] each."""
    V = logits.shape[1]
    out = [np.full((G, n), -np.inf), np.full((G, n), -1), np.full((G, n), -1), np.ones((G, n), dtype=int)]
    for g in range(G):
        found = []
        for r in range(g * K, g * K + K):
            s = float(scores[r])
            if not math.isfinite(s):
                continue
            if finished is not None and finished[r]:
                found.append((-s, r, -1))
                continue
            ok = np.ones(V, dtype=bool) if allowed is None else allowed[r]
            total, infinite = log_total(logits[r], np.ones(V, dtype=bool) if over_all else ok)
            ids = np.flatnonzero(ok & ~np.isnan(logits[r]) & (np.isposinf(logits[r]) if infinite else logits[r] != -np.inf))
            if not len(ids):
                continue
            value = (0.0 if infinite else logits[r][ids].astype(np.float64)) + np.full(len(ids), s - total)
            if len(ids) > n:
                keep = value >= np.partition(value, len(ids) - n)[len(ids) - n]
                ids, value = ids[keep], value[keep]
            found += [(-v, r, int(t)) for v, t in zip(value.tolist(), ids)]
        for j, (v, r, t) in enumerate(sorted(found)[:n]):
            out[0][g, j], out[1][g, j], out[2][g, j], out[3][g, j] = -v, r, t, int(t < 0 or t == eos)
    return out


def score_tolerance(V, score):
    """A chosen score is off by the row's sum, taken in 32 bits, and by one rounding to 32 bits at the end.  The sum, relative to its
    value: a term exp2(t), t = x log2(e) - c, is off by one unit of exp2 (2^-23) and by the rounding of t (|t| 2^-24 ln 2 = (top - x)
    2^-24; its mean over the probabilities is at most ln V); 11 additions lie between a term and its piece's sum (2^-24 each)."""
    return (math.log(max(V, 2)) + 2 + 11) * 2.0 ** -24 + np.abs(score) * 2.0 ** -24


def reorder(state, parents, G, K):
    """New list of states by the parents of each group; a parent of -1 or outside the group keeps the state."""
    out = list(state)
    for r in range(G * K):
        p = int(parents[r])
        if r // K * K <= p < r // K * K + K:
            out[r] = state[p]
    return out


def backtrace(tokens, parents, G, K):
    T, R = tokens.shape
    out, length = np.full((R, T), -1, dtype=np.int32), np.zeros(R, dtype=np.int32)
    for r in range(R):
        at, g = r, r // K
        for t in range(T - 1, -1, -1):
            out[r, t] = tokens[t, at]
            at = int(parents[t, at])
            if not g * K <= at < g * K + K:
                break
        seen = np.flatnonzero(out[r] >= 0)
        length[r] = seen[-1] + 1 if len(seen) else 0
    return out, length
