"""Rows of a paged cache made for the tests of the softmax's weights: a pool from given keys and values, and the bound of an output whose values are all
of one sign (no GPU, nothing of the library but its codec's models)."""
from __future__ import annotations

import numpy as np

EPS32, EPS16 = 2.0 ** -24, 2.0 ** -11  # half a step of FP32 and FP16, relative


def pool(oracle, models, keys, values, page, seed):
    """keys, values: per sequence [tokens, heads, 128] FP16.  (table, the four arrays of the pool, decoded keys, decoded values); pages in
    random order, blocks that hold no token full of ones."""
    rng = np.random.default_rng(seed)
    heads, lens = keys[0].shape[1], [len(k) for k in keys]
    n = [-(-t // page) for t in lens]
    order, at = rng.permutation(sum(n) + 2), 0
    table = np.full((len(lens), max(n) + 1), 2 ** 31 - 1)
    arrays = [np.full((len(order), heads, page, 64), 255, np.uint8), np.full((len(order), heads, page), -1, np.int32)] * 2
    arrays = [a.copy() for a in arrays]
    decoded = [[], []]
    for b, t in enumerate(lens):
        table[b, :n[b]] = order[at:at + n[b]]
        at += n[b]
        pages, off = np.repeat(table[b, :n[b]], page)[:t], np.tile(np.arange(page), n[b])[:t]
        for i, (x, m) in enumerate(zip((keys[b], values[b]), models)):
            blocks, meta = oracle.encode(m.centroids, m.code_lens, np.ascontiguousarray(x).reshape(-1, 128).view(np.uint16))
            arrays[2 * i][pages, :, off] = blocks.reshape(t, heads, 64)
            arrays[2 * i + 1][pages, :, off] = meta.view(np.int32).reshape(t, heads)
            decoded[i].append(oracle.decode(m.centroids, m.code_lens, blocks, meta).view(np.float16).reshape(t, heads, 128))
    return table, arrays, decoded[0], decoded[1]


def attend(q, keys, values, seen, half, few):
    """One sequence and key/value head in 64 bits, values not negative: (outputs, bound of each element), q [rows, 128], seen [rows, tokens].

    All terms of numerator and denominator are of one sign, so what is relative to a term is relative to the sum:
      score   a sum of 128 products in FP32 is off by at most 130 half steps of a = sum |q k| / sqrt(128), scaling included; two scores
      exp     its argument, at most 2 a and 15 binary places of a common factor, is off by 4 half steps of either; itself by 4 half steps
      weight  as two FP16 numbers 2^-22, as one (FP16 outputs, many rows) half a step, 2^-11; or, whatever its size, half of FP16's least step
              below the largest weight's place, which is 2^11 at the least: 2^-36 of the largest weight
      sums    half a step per token
    of the numerator and the denominator each; and half a step of the result, FP16's least step where it is subnormal."""
    q, keys, values = (np.asarray(a, np.float64) for a in (q, keys, values))
    assert (values >= 0).all()
    score = q @ keys.T / np.sqrt(128.0)
    size = np.where(seen, np.abs(q) @ np.abs(keys).T / np.sqrt(128.0), 0.0).max(1)
    top = np.where(seen, score, -np.inf).max(1, keepdims=True)
    p = np.where(seen, np.exp(np.where(seen, score - top, 0.0)), 0.0)
    out = p @ values / p.sum(1, keepdims=True)
    n = seen.sum(1)
    rel = 2 * (2 * 130 * EPS32 * size + 4 * EPS32 * (2 * size + 15) + 4 * EPS32 + n * EPS32) + (2.0 ** -22 if few or not half else EPS16) + 4 * EPS32
    bound = rel[:, None] * out + (n * 2.0 ** -36)[:, None] * values.max(0)
    if half:
        bound = bound + EPS16 * (out + bound) + 2.0 ** -25
    return out, bound
