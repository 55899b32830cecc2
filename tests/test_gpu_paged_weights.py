"""Attention over pages where small weights matter: a row whose first token leads by far and has a small value, before thousands of tokens far behind it whose
values add up.  Every weight has to keep its bits, whatever its size beside the largest."""
from __future__ import annotations

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2505_06901_amd as E  # noqa: E402

import paged_rows as P  # noqa: E402

LEADS = (2.0, 9.0, 12.0, 14.5, 16.0, 17.5, 19.0, 24.0)  # by how much the first token is ahead, in powers of e


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


@pytest.fixture(scope="module")
def models(dev):
    rng = np.random.default_rng(1)
    return [E.ecco_model_to_device(E.ecco_fit_patterns(x.astype(np.float16), 16, 12, 5), 0)
            for x in (rng.standard_normal((512, 128)), rng.uniform(0.5, 1.5, (512, 128)))]


def _sequence(tokens, heads, seed):
    """Keys: the first one along a direction of ones, the others small and at random; values: the first one 2^-12, the others 0.5 to 1.5."""
    rng = np.random.default_rng(seed)
    k, v = 0.02 * rng.standard_normal((tokens, heads, 128)), rng.uniform(0.5, 1.5, (tokens, heads, 128))
    k[0], v[0] = rng.uniform(0.8, 1.0, (heads, 128)), rng.uniform(0.5, 1.5, (heads, 128)) * 2.0 ** -12
    return k.astype(np.float16), v.astype(np.float16)


def _queries(rows, Hq, leads):
    """Along the same direction, each query with its own lead: the first key's product with the direction is 128 * 0.9."""
    lead = np.resize(leads, rows * Hq).reshape(rows, Hq, 1)
    return np.broadcast_to(lead * np.sqrt(128.0) / (128 * 0.9), (rows, Hq, 128)).astype(np.float16)


CASES = [
    # Hq, Hkv, page, [(new, kv)]
    (8, 2, 16, [(1, 9000)]),                       # up to 8 rows, ranges
    (4, 1, 64, [(1, 200)]),                        # one range
    (16, 16, 32, [(1, 700)] * 17),                 # a workgroup per sequence and head, several spans
    (8, 2, 32, [(3, 5000), (2, 40)]),              # up to 16 rows
    (16, 2, 16, [(4, 9000)]),                      # up to 32 rows
    (4, 1, 16, [(1, 3000), (40, 9000)]),           # tiles of 128 rows, ranges
    (8, 8, 32, [(260, 1500)] * 16),                # tiles of 128 rows, whole
    (128, 8, 64, [(790, 3200)]),                   # tiles of 256 rows
]


def _check(dev, oracle, models, case, half, leads, seed):
    Hq, Hkv, page, spans = CASES[case]
    new, kv = [n for n, _ in spans], [t for _, t in spans]
    grp = Hq // Hkv
    data = [_sequence(t, Hkv, seed + b % 3) for b, t in enumerate(kv)]
    table, arrays, keys, values = P.pool(oracle, models, [k for k, _ in data], [v for _, v in data], page, seed)
    q = _queries(sum(new), Hq, leads)
    ints = lambda a: torch.from_numpy(np.asarray(a, np.int32)).to(dev)  # noqa: E731
    pool = [torch.from_numpy(a).to(dev) for a in arrays]
    out = torch.empty(q.shape, dtype=torch.float16 if half else torch.float32, device=dev)
    E.ecco_kv_attend_paged(*models, torch.from_numpy(q).to(dev), *pool, ints(table), ints(np.concatenate([[0], np.cumsum(new)])), ints(kv), max(new), max(kv), sum(kv),
                           out=out)
    got, row = out.cpu().numpy().astype(np.float64), 0
    for b, (n, t) in enumerate(spans):
        for h in range(Hkv) if b < 3 else ():  # (the sequences' keys and values repeat)
            few = n * grp <= (32 if max(new) * grp <= 32 else grp)
            pick = np.unique(np.concatenate([np.arange(min(n, 8)), np.arange(max(n - 8, 0), n)]))  # the first and the last rows, every lead
            seen = np.repeat(np.arange(t)[None, :] <= (t - n + pick)[:, None], grp, 0)
            o, bound = P.attend(q[row + pick, h * grp:(h + 1) * grp].reshape(-1, 128), keys[b][:, h], values[b][:, h], seen, half, few)
            err = np.abs(got[row + pick, h * grp:(h + 1) * grp].reshape(-1, 128) - o)
            worst = np.unravel_index(np.argmax(err / bound), err.shape)
            assert (err <= bound).all(), (CASES[case], b, h, worst, err[worst], bound[worst], o[worst])
        row += n


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("case", range(5))
def test_small_weights_few_rows(dev, oracle, models, case, half):
    _check(dev, oracle, models, case, half, LEADS, 100 + case)


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("case", range(5, 8))
def test_small_weights_many_rows(dev, oracle, models, case, half):
    _check(dev, oracle, models, case, half, LEADS, 200 + case)


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("case", [0, 5])
def test_a_lead_that_comes_late(dev, oracle, models, case, half):
    """The other way round: leads below zero put the first token behind all others, so that it does not weigh at all and the rest is a mean."""
    _check(dev, oracle, models, case, half, (-20.0, -3.0, 0.0, 1.0), 300 + case)
