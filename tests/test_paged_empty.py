"""Steps over pages that have nothing to do (no GPU): they are not refused for their sizes."""
from __future__ import annotations

import pytest

import paper_2505_06901_amd as E
from paper_2505_06901_amd import binding, workloads as W

from test_paged_host import ATTEND, EINVAL, ESHAPE


@pytest.fixture(scope="module")
def model():
    return E.ecco_fit_patterns(W.config_weight("tiny"), 16, 12, 0)


def _attend(model, **changed):
    return binding.lib().ecco_kv_attend_paged(*dict(ATTEND, mk=model.handle, mv=model.handle, **changed).values())


@pytest.mark.parametrize("none", [dict(), dict(B=0), dict(max_new=0), dict(max_kv=0), dict(total_kv=0), dict(B=0, max_new=0, max_kv=0, total_kv=0)])
def test_a_step_without_rows_gets_past_the_sizes(model, none):
    """... as far as the models, which are on no device here: the last check."""
    assert _attend(model, n_tokens=0, **none) == EINVAL
    if none:
        assert _attend(model, **none) == ESHAPE


@pytest.mark.parametrize("bad", [dict(B=-1), dict(max_new=-1), dict(max_kv=-1), dict(total_kv=-1), dict(Hq=0), dict(Hkv=0), dict(page_tokens=8), dict(n_pages=0), dict(max_pages=0)])
def test_a_step_without_rows_still_needs_sizes(model, bad):
    assert _attend(model, n_tokens=0, **bad) == ESHAPE
