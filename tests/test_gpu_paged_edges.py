"""The paged cache's calls that the documentation allows and that ordinary use makes seldom."""
from __future__ import annotations

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2505_06901_amd as E  # noqa: E402
from paper_2505_06901_amd import workloads as W  # noqa: E402

import paged_reference as R  # noqa: E402
import paged_rows as P  # noqa: E402


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


@pytest.fixture(scope="module")
def models(dev):
    k, v = W.kv_cache(1, 4, 192, 128, seed=3)
    return [E.ecco_model_to_device(E.ecco_fit_patterns(x, 16, 12, 5), 0) for x in (k, v)]


def ints(a, dev):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(dev)


class Cache:
    """A pool of sequences of the given lengths, with what they decode to."""

    def __init__(self, dev, oracle, models, lens, heads, page, seed):
        data = [W.kv_cache(1, heads, t, 128, seed=seed + b) for b, t in enumerate(lens)]
        self.heads, self.models = heads, models
        table, arrays, self.keys, self.values = P.pool(oracle, models, [k[0].transpose(1, 0, 2) for k, _ in data], [v[0].transpose(1, 0, 2) for _, v in data], page, seed)
        self.table, self.pool = ints(table, dev), [torch.from_numpy(a).to(dev) for a in arrays]

    def want(self, q, b, n, kv):
        """Outputs and bounds of sequence b's n rows q [n, Hq, 128] over its first kv tokens."""
        grp, out, bound = q.shape[1] // self.heads, np.zeros(q.shape), np.zeros(q.shape)
        seen = np.repeat(np.arange(kv)[None, :] <= (kv - n + np.arange(n))[:, None], grp, 0)
        for h in range(self.heads):
            at = np.s_[:, h * grp:(h + 1) * grp]
            o, e = R.attend(q[at].reshape(-1, 128), self.keys[b][:kv, h], self.values[b][:kv, h], seen)
            out[at], bound[at] = o.reshape(n, grp, 128), e.reshape(n, grp, 128)
        return out, bound


def queries(rows, Hq, seed):
    return W.activation(rows * Hq, 128, seed).reshape(rows, Hq, 128)


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("what", [float("nan"), float("inf")])
@pytest.mark.parametrize("Hq,Hkv,spans", [
    (8, 2, [(1, 200), (1, 90)]),            # up to 8 rows, one range
    (8, 2, [(1, 3000), (2, 200)]),          # ranges
    (16, 2, [(2, 700), (1, 300)]),          # up to 16 rows
    (16, 2, [(4, 200), (3, 2000)]),         # up to 32 rows
    (16, 2, [(70, 600), (1, 500)]),         # tiles, ranges
    (8, 2, [(160, 400)] * 13),              # tiles, whole
    (128, 8, [(790, 800)]),                 # tiles of 256 rows
])
def test_queries_that_are_not_finite_reach_their_own_outputs_only(dev, oracle, models, Hq, Hkv, spans, what, half):
    new, kv = [n for n, _ in spans], [t for _, t in spans]
    c = Cache(dev, oracle, models, kv, Hkv, 16, 10)
    q = torch.from_numpy(queries(sum(new), Hq, 11)).to(dev)
    call = lambda: E.ecco_kv_attend_paged(*models, q, *c.pool, c.table, ints(np.concatenate([[0], np.cumsum(new)]), dev), ints(kv, dev), max(new), max(kv), sum(kv),  # noqa: E731
                                          out=torch.empty(q.shape, dtype=torch.float16 if half else torch.float32, device=dev))
    clean = call()
    at = [(0, 0, 5), (sum(new) - 1, Hq - 1, 127), (new[0] - 1, Hq // 2, 0)]
    for r, h, d in at:
        q[r, h, d] = what
    got = call()
    bad = torch.zeros(q.shape[:2], dtype=torch.bool, device=dev)
    for r, h, _ in at:
        bad[r, h] = True
    assert torch.isnan(got[bad]).all()
    # the others may be scaled at other moments: the same but for the last bits
    assert torch.allclose(got[~bad].float(), clean[~bad].float(), rtol=0, atol=float(clean.float().abs().max()) * (2.0 ** -10 if half else 2.0 ** -18))
