"""The operators of the paged cache from their definitions, in plain Python and 64 bits, for the tests (no GPU, nothing of the library)."""
from __future__ import annotations

import numpy as np

EPS32, EPS16 = 2.0 ** -24, 2.0 ** -11  # half a step of FP32 and FP16, relative


def take(seq_len, new_len, table, free, count, page, n_tokens):
    """(table, pages left, q_start, kv_len, slots); table [B][max_pages], free: the stack."""
    table, n_pages, max_pages = np.array(table, np.int64), len(free), np.shape(table)[1]
    count = min(max(int(count), 0), n_pages)
    rows = asked = gone = 0
    starts, lens, slots = [0], [], np.full(n_tokens, -1, np.int64)
    for b, (held, new) in enumerate(zip(seq_len, new_len)):
        held, new = max(int(held), 0), max(int(new), 0)
        have, want = -(-held // page), -(-(held + new) // page)
        served = rows + new <= n_tokens and want <= max_pages
        if served:
            asked += want - have
            served = want == have or asked <= count
        if served:
            for i in range(have, want):
                gone += 1
                table[b, i] = free[count - gone]
            for i, t in enumerate(range(held, held + new)):
                at = table[b, t // page]
                if 0 <= at < n_pages:
                    slots[rows + i] = at * page + t % page
        rows += new
        starts.append(min(rows, n_tokens))
        lens.append(held + new if served else 0)
    return table, count - gone, np.array(starts), np.array(lens), slots


def release(seq_len, keep_len, table, free, count, page):
    """(stack, pages on it)."""
    free, n_pages, max_pages = np.array(free, np.int64), len(free), np.shape(table)[1]
    count = min(max(int(count), 0), n_pages)
    for row, held, keep in zip(np.asarray(table), seq_len, keep_len):
        held = max(int(held), 0)
        keep = min(max(int(keep), 0), held)
        for i in range(-(-keep // page), min(-(-held // page), max_pages)):
            if 0 <= row[i] < n_pages and count < n_pages:
                free[count] = row[i]
                count += 1
    return free, count


def attend(q, keys, values, seen):
    """One sequence and key/value head in 64 bits: q [rows, 128], keys, values [tokens, 128], seen [rows, tokens].  (outputs, bounds): the
    bound of an element is what rounding can make of it in FP32:
      score   a sum of 128 products in FP32 is off by at most 130 half steps of a = sum |q k| / sqrt(128), scaling included
      exp     of s - m, at most 2 a in size: off by its argument's error (both scores', and the product with log2(e): 4 half steps
              of 2 a) and its own (4 half steps, 2 ulp)
      sums    of the weights and of weight times value: half a step per token each, plus 2^-22 for a weight held as two FP16 numbers (and
              2^-24 of the largest weight for a rest below FP16's normal range)
    all relative to the largest |value| of the dimension, numerator and denominator alike."""
    q, keys, values = (np.asarray(a, np.float64) for a in (q, keys, values))
    score = q @ keys.T / np.sqrt(128.0)
    size = np.where(seen, np.abs(q) @ np.abs(keys).T / np.sqrt(128.0), 0.0).max(1, initial=0.0)
    any_seen = seen.any(1)
    top = np.where(seen, score, -np.inf).max(1, initial=-np.inf, keepdims=True)
    p = np.where(seen, np.exp(np.where(seen, score - np.where(any_seen[:, None], top, 0.0), 0.0)), 0.0)
    den = p.sum(1, keepdims=True)
    out = np.where(any_seen[:, None], p @ values / np.where(den > 0, den, 1.0), 0.0)
    n = seen.sum(1)
    weight = 2 * 130 * EPS32 * size + 8 * EPS32 * size + 4 * EPS32
    rel = 2 * (weight + n * EPS32) + 2.0 ** -22 + n * 2.0 ** -24 * 2.0 ** -10 + 8 * EPS32
    most = np.array([np.abs(values[s]).max(0, initial=0.0) for s in seen]).reshape(len(q), 128)
    return out, rel[:, None] * most


def check_attend(got, want, bound, half, tag=None):
    """Element by element against the bound; for FP16 outputs half a step of the result and, where probabilities enter the product as one FP16
    number, half a step of each of them (numerator and denominator) on top.  And as norms over the rows: the errors of the products and sums
    are not all of one sign, so that the norm of 128 elements stays within a sixteenth of their bounds (roundings of both signs add up as the
    root of their number: 130 of them as 11)."""
    got = np.asarray(got, np.float64)
    if not got.size:
        return
    assert np.isfinite(got).all(), tag
    err = np.abs(got - want)
    extra = 2 * EPS16 * np.abs(want) + 2.0 ** -24 + 2 * EPS16 * bound["most"] if half else 0.0
    worst = np.unravel_index(np.argmax(err - bound["element"] - extra), err.shape)
    assert (err <= bound["element"] + extra).all(), (tag, worst, err[worst], bound["element"][worst])
    norm = np.linalg.norm(err, axis=-1)
    limit = np.linalg.norm(bound["element"], axis=-1) / 16 + (np.linalg.norm(extra, axis=-1) if half else 0.0)
    assert (norm <= limit).all(), (tag, np.unravel_index(np.argmax(norm - limit), norm.shape), norm.max(), limit.min())
