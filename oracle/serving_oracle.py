"""The slow CPU definition of the serving calls (prompts of any length, a cache of pages, attention of single tokens), in numpy
and 64 bits.  Test infrastructure only.

Bounds.  What the kernels may differ by follows from their arithmetic (`bound`): with eps = 2^-8, half a step of bf16 relative
to the value,
  O    the result is rounded to bf16: eps |O|; the probabilities are, before they multiply V: eps A, where A is the average of
       |v| under the probabilities; where the sum of the rounded ones divides, it moves by another eps |O|
  x    a logit is a sum of 128 products in fp32, scaled, and its exponential one in fp32: an error of at most `slack` in the
       exponent, 2^-17 of |q| |k| / sqrt(d) (128 additions of relative error 2^-24) plus 2^-19; it enters O twice (value, sum)
  lse  `slack` and the rounding of a number of its own size in fp32 (the prompt call sums rounded probabilities: 2^-8 more)
"""
from __future__ import annotations

import numpy as np

EPS = 2.0 ** -8


def attend(q, k, v, seen):
    """q [rows, d], k, v [keys, d] in 64 bits, seen [rows, keys] bool -> O, lse, bound of O, slack of the logits.  Rows that see no
    key: O = 0, lse = -inf.  What a row does not see has no effect on it, whatever it is."""
    rows, d = q.shape
    o, lse = np.zeros((rows, v.shape[1])), np.full(rows, -np.inf)
    tol, slack = np.zeros((rows, v.shape[1])), np.zeros(rows)
    for r in range(rows):
        ks, vs = k[seen[r]], v[seen[r]]
        if len(ks) == 0:
            continue
        with np.errstate(invalid="ignore", over="ignore"):
            x = ks @ q[r] / np.sqrt(d)
            top = x.max()
            e = np.exp(x - top)
            total = e.sum()
            o[r] = (e[:, None] * vs).sum(axis=0) / total
            lse[r] = top + np.log(total)
            a = (e[:, None] * np.abs(vs)).sum(axis=0) / total
            slack[r] = 2.0 ** -17 * np.sqrt((q[r] ** 2).sum() * (ks ** 2).sum(axis=1).max()) / np.sqrt(d) + 2.0 ** -19
            tol[r] = EPS * (2 * np.abs(o[r]) + a) + 2 * slack[r] * a + 1e-30
    return o, lse, tol, slack


def prompt(q, k, v, offsets):
    """q [Hq, N, d], k, v [Hkv, N, d] in 64 bits; offsets of the packed sequences -> O, lse, bound of O, slack, [Hq, N, ..]."""
    hq, n, d = q.shape
    group = hq // k.shape[0]
    out = [np.zeros(q.shape), np.full((hq, n), -np.inf), np.zeros(q.shape), np.zeros((hq, n))]
    for t0, t1 in zip(offsets[:-1], offsets[1:]):
        seen = np.tril(np.ones((t1 - t0, t1 - t0), dtype=bool))
        for h in range(hq):
            for into, got in zip(out, attend(q[h, t0:t1], k[h // group, t0:t1], v[h // group, t0:t1], seen)):
                into[h, t0:t1] = got
    return out


def decode(q, k_pages, v_pages, table, lens, prefix_pages, prefix_len):
    """q [S, Hq, n, d]; pages [P, Hkv, T, d], all in 64 bits (8-bit ones times their scales); table [S, W], lens [S] -> as prompt."""
    n_seqs, hq, n, d = q.shape
    n_pages, hkv, page, _ = k_pages.shape
    group = hq // hkv
    out = [np.zeros(q.shape), np.full(q.shape[:3], -np.inf), np.zeros(q.shape), np.zeros(q.shape[:3])]

    def keys(pages, entries, count):
        """Positions 0 .. count - 1 of a list of pages: [Hkv, count, d], and whether there is a key."""
        x, there = np.zeros((hkv, count, d)), np.zeros(count, dtype=bool)
        for i in range(count):
            e = int(entries[i // page])
            if 0 <= e < n_pages:
                x[:, i], there[i] = pages[e][:, i % page], True
        return x, there

    for s in range(n_seqs):
        count = min(max(int(lens[s]), 0), table.shape[1] * page)
        shared = [keys(x, prefix_pages, prefix_len) for x in (k_pages, v_pages)]
        own = [keys(x, table[s], count) for x in (k_pages, v_pages)]
        k, v = (np.concatenate([a[0], b[0]], axis=1) for a, b in zip(shared, own))
        there = np.concatenate([shared[0][1], own[0][1]])
        at = np.concatenate([np.full(prefix_len, -1), np.arange(count)])
        seen = np.stack([there & (at <= max(int(lens[s]), 0) - n + t) | there & (at < 0) for t in range(n)])
        for h in range(hq):
            for into, got in zip(out, attend(q[s, h], k[h // group], v[h // group], seen)):
                into[s, h] = got
    return out


def positions(lens, new):
    """(sequence, token among its new ones, position) of every new token that has a position."""
    return [(s, i, max(int(lens[s]), 0) - n + i) for s, n in enumerate(new) for i in range(n) if max(int(lens[s]), 0) - n + i >= 0]


def e4m3(x):
    """The value of OCP E4M3 nearest to x (fp32 or 64 bits), ties to even, at most 448 in size; NaN stays."""
    x = np.asarray(x, dtype=np.float64)
    with np.errstate(invalid="ignore", divide="ignore"):
        step = np.exp2(np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -6))) - 3)
        return np.where(np.isnan(x), np.nan, np.clip(np.where(np.isinf(x), x, np.round(x / step) * step), -448.0, 448.0))
