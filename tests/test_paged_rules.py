"""What a program has to keep to that strings steps over pages together, followed in the plain definitions (no GPU): how lengths advance."""
from __future__ import annotations

import numpy as np
import pytest

import paged_reference as R


def _serve(advance, seed, steps=60):
    """Sequences that grow until pages run out, end now and then and give their pages back.  (pages that are on the stack once all have ended, pages;
    whether a token's slot was ever one that another sequence holds)."""
    rng = np.random.default_rng(seed)
    page, n_pages, B, max_pages = 16, 12, 4, 8
    lens, table, free, count = np.zeros(B, np.int64), np.full((B, max_pages), -1), rng.permutation(n_pages), n_pages
    owner, clash = {}, False
    for _ in range(steps):
        new = rng.integers(0, 30, B)
        table, count, q_start, kv, slots = R.take(lens, new, table, free, count, page, int(new.sum()))
        for b in range(B):
            for i in range(new[b]):
                slot = int(slots[q_start[b] + i])
                if slot >= 0:
                    at = (b, int(lens[b]) + i)
                    clash |= owner.get(slot, at)[0] != b
                    owner[slot] = at
        lens = advance(lens, kv)
        done = rng.random(B) < 0.15
        free, count = R.release(lens, np.where(done, 0, lens), table, free, count, page)
        owner = {s: o for s, o in owner.items() if not done[o[0]]}
        lens = np.where(done, 0, lens)
    free, count = R.release(lens, np.zeros(B), table, free, count, page)
    return sorted(free[:count].tolist()), list(range(n_pages)), clash


@pytest.mark.parametrize("seed", range(5))
def test_lengths_advance_to_the_larger_of_both(seed):
    back, pages, clash = _serve(np.maximum, seed)
    assert back == pages and not clash


def test_lengths_do_not_advance_to_kv_len_alone():
    """The same with kv_len for the length: sequences that were not served lose their pages."""
    assert any(_serve(lambda lens, kv: kv, seed)[0] != list(range(12)) for seed in range(5))
