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


def test_captured_steps_that_run_out_of_pages(dev, oracle, models):
    """A whole step in a graph whose sequences grow until pages run out: those that are not served give zeros, keep their length, pages and tokens, and go on once
    others have ended; at the end every page is back."""
    B, Hq, Hkv, page, n_pages, max_pages, n_new = 4, 8, 2, 16, 9, 6, 5
    rng = np.random.default_rng(8)
    table, free, count, lens = ints(np.full((B, max_pages), -1), dev), ints(rng.permutation(n_pages), dev), ints([n_pages], dev), ints(np.zeros(B), dev)
    pool = [torch.zeros((n_pages, Hkv, page, 64), dtype=torch.uint8, device=dev), torch.zeros((n_pages, Hkv, page), dtype=torch.int32, device=dev)] * 2
    pool = [t.clone() for t in pool]
    rows, new = B * n_new, ints(np.full(B, n_new), dev)
    q, k, v = (torch.zeros((rows, h, 128), dtype=torch.float16, device=dev) for h in (Hq, Hkv, Hkv))
    out, kv_len = torch.empty((rows, Hq, 128), dtype=torch.float32, device=dev), ints(np.zeros(B), dev)

    def step():
        q_start, _, slots = E.ecco_kv_pages_take(lens, new, table, free, count, page, rows, kv_len=kv_len)
        E.ecco_kv_append_paged(*models, k, v, *pool, slots)
        E.ecco_kv_attend_paged(*models, q, *pool, table, q_start, kv_len, n_new, max_pages * page, out=out)
        torch.maximum(lens, kv_len, out=lens)

    new.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()  # (no new tokens: nothing changes)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    keys, values = [np.zeros((0, Hkv, 128), np.float16)] * B, [np.zeros((0, Hkv, 128), np.float16)] * B
    decoded = lambda m, x: oracle.decode(m.centroids, m.code_lens, *oracle.encode(m.centroids, m.code_lens, x.reshape(-1, 128).view(np.uint16))).view(np.float16).reshape(x.shape)  # noqa: E731
    refused = 0
    for i in range(16):
        count_new = rng.integers(0, n_new + 1, B) if i % 3 else np.full(B, n_new)
        n = int(count_new.sum())
        qh, (kh, vh) = queries(rows, Hq, 40 + i), (np.ascontiguousarray(x[0].transpose(1, 0, 2)) for x in W.kv_cache(1, Hkv, rows, 128, seed=60 + i))
        for t, x in ((q, qh), (k, kh), (v, vh)):
            t.copy_(torch.from_numpy(x))
        new.copy_(ints(count_new, dev))
        graph.replay()
        torch.cuda.synchronize()
        got, kv, row = out.cpu().numpy(), kv_len.cpu().numpy(), 0
        for b, m in enumerate(count_new):
            at = np.s_[row:row + m]
            row += m
            if kv[b] == 0 and len(keys[b]) + m > 0:  # not served
                refused += 1
                assert not got[at].any()
                continue
            if m:
                keys[b], values[b] = np.concatenate([keys[b], decoded(models[0], kh[at])]), np.concatenate([values[b], decoded(models[1], vh[at])])
            assert kv[b] == len(keys[b])
            seen = np.repeat(np.arange(kv[b])[None, :] <= (kv[b] - m + np.arange(m))[:, None], Hq // Hkv, 0)
            for h in range(Hkv):
                o, e = R.attend(qh[at, h * 4:h * 4 + 4].reshape(-1, 128), keys[b][:, h], values[b][:, h], seen)
                R.check_attend(got[at, h * 4:h * 4 + 4].reshape(-1, 128), o, {"element": e, "most": 0.0}, False, (i, b, h))
        assert row == n and lens.tolist() == [len(x) for x in keys], i
        if i % 5 == 4:  # the longest one has ended
            b = int(np.argmax([len(x) for x in keys]))
            keep = [0 if j == b else len(x) for j, x in enumerate(keys)]
            E.ecco_kv_pages_release(lens, ints(keep, dev), table, free, count, page)
            lens.copy_(ints(keep, dev))
            keys[b], values[b] = keys[b][:0], values[b][:0]
    assert refused > 0  # (the path was reached)
    E.ecco_kv_pages_release(lens, ints(np.zeros(B), dev), table, free, count, page)
    assert int(count) == n_pages and sorted(free.tolist()) == list(range(n_pages))


@pytest.mark.parametrize("half", [False, True])
def test_one_workspace_for_every_step(dev, oracle, models, half):
    """A workspace allocated for the largest step, and nothing behind it written, serves steps that are planned in other ways: ranges, none, splits, tiles of 256."""
    Hq, Hkv, lens = 128, 8, [2100, 900, 40] + [70] * 29
    c = Cache(dev, oracle, models, lens, Hkv, 16, 20)
    steps = [[1] * 32, [1] * 31, [1, 1, 1], [2, 2, 1], [64, 1, 1], [800, 300, 40], [2, 900], [1] + [0] * 31, [1200, 1, 0, 3]]
    largest = E.ecco_kv_attend_paged_workspace(1300, 32, Hq, Hkv, 1200, 2100, sum(lens))
    memory = torch.full((largest + 4096,), 0xA5, dtype=torch.uint8, device=dev)
    for i, new in enumerate(steps):
        kv = lens[:len(new)]
        q = torch.from_numpy(queries(sum(new), Hq, 30 + i)).to(dev)
        args = (*models, q, *c.pool, c.table[:len(new)].contiguous(), ints(np.concatenate([[0], np.cumsum(new)]), dev), ints(kv, dev), max(new), max(kv), sum(kv))
        out = [torch.empty(q.shape, dtype=torch.float16 if half else torch.float32, device=dev) for _ in range(2)]
        E.ecco_kv_attend_paged(*args, workspace=memory[:largest], out=out[0])
        E.ecco_kv_attend_paged(*args, out=out[1])
        assert torch.equal(*out) and torch.isfinite(out[0]).all(), new
        assert bool((memory[largest:] == 0xA5).all()), new


def test_a_step_without_rows(dev, models):
    pool = [torch.zeros((3, 2, 16, 64), dtype=torch.uint8, device=dev), torch.zeros((3, 2, 16), dtype=torch.int32, device=dev)] * 2
    q = torch.zeros((0, 8, 128), dtype=torch.float16, device=dev)
    for B in (0, 2):
        out = E.ecco_kv_attend_paged(*models, q, *pool, ints(np.zeros((B, 4)), dev), ints(np.zeros(B + 1), dev), ints(np.zeros(B), dev), 0, 0)
        assert out.shape == q.shape


@pytest.mark.parametrize("B,new,kv,bounds,fits", [
    # (max_new, max_kv, total_kv) that the lengths exceed; how many sequences come before the first that does not fit
    (6, 40, 300, (40, 300, 700), 2),          # 21 + 6 units of 32 tokens for ten each
    (6, 40, 300, (40, 300, 1), 0),            # six for ten
    (130, 9, 200, (9, 200, 1), 18),           # 130 units for seven each; the layout in a launch of its own
    (130, 9, 200, (9, 200, 12800), 75),       # 400 + 130: the first that does not fit is in the second set of 64
    (2, (40, 260), 90, (40, 90, 180), 1),     # four tiles for two and nine
    (66, (9,) * 65 + (130,), 40, (9, 40, 66 * 40), 65),  # as many tiles as sequences
])
@pytest.mark.parametrize("half", [False, True])
def test_many_rows_beyond_the_bounds(dev, oracle, models, B, new, kv, bounds, fits, half):
    """Lengths on the device that need more of the workspace or the launch than the bounds provide: sequences ahead of the first that does not fit are what they
    are, it and those behind it are left unwritten, and so is what lies behind the workspace."""
    Hq, Hkv, new = 8, 2, [new] * B if isinstance(new, int) else list(new)
    c = Cache(dev, oracle, models, [kv] * B, Hkv, 16, 50)
    n, guard = sum(new), 1 << 20
    q = queries(n, Hq, 51)
    size = E.ecco_kv_attend_paged_workspace(n, B, Hq, Hkv, *bounds)
    memory = torch.full((size + guard,), 0xA5, dtype=torch.uint8, device=dev)
    out = torch.full((n + 4, Hq, 128), float("nan"), dtype=torch.float16 if half else torch.float32, device=dev)
    E.ecco_kv_attend_paged(*models, torch.from_numpy(q).to(dev), *c.pool, c.table, ints(np.concatenate([[0], np.cumsum(new)]), dev), ints([kv] * B, dev), *bounds, memory[:size], out[:n])
    got, row = out.cpu().numpy(), 0
    assert bool((memory[size:] == 0xA5).all())
    for b in range(fits):
        if b % 8 == 0 or b >= fits - 2:
            want, bound = c.want(q[row:row + new[b]], b, new[b], kv)
            R.check_attend(got[row:row + new[b]], want, {"element": bound, "most": float(np.abs(c.values[b].astype(np.float64)).max())}, half, b)
        row += new[b]
    assert np.isfinite(got[:row]).all() and np.isnan(got[row:]).all()


@pytest.mark.parametrize("starts,lens,whole", [
    ([0, 1, 3, 4], [300, 2 ** 31 - 1, 100], {0: (0, 1), 2: (3, 4)}),    # a length behind max_kv: its sequence sees what lies there
    ([0, 1, 3, 2 ** 31 - 1], [300, 500, -4], {0: (0, 1), 1: (1, 3)}),   # rows behind n_tokens: none
    ([0, 1, -7, 1], [300, 500, 100], {0: (0, 1)}),                      # starts that do not ascend: none
    ([0, 1, 3, 4], [300, 500, -4], {0: (0, 1), 1: (1, 3), 2: (3, 4)}),  # a negative length: sees nothing
])
def test_few_rows_beyond_the_bounds(dev, oracle, models, starts, lens, whole):
    """Every row that the bounds cover is what it is, and rows of no sequence are left as they were."""
    kv = [300, 500, 100]
    c = Cache(dev, oracle, models, kv, 2, 16, 60)
    q = queries(4, 8, 61)
    out = torch.full((6, 8, 128), float("nan"), dtype=torch.float32, device=dev)
    E.ecco_kv_attend_paged(*models, torch.from_numpy(q).to(dev), *c.pool, c.table, ints(starts, dev), ints(lens, dev), 2, 512, 900, out=out[:4])
    got, rows = out.cpu().numpy(), set(range(6))
    for b, (i, j) in whole.items():
        t = max(min(lens[b], kv[b]), 0)
        want, bound = c.want(q[i:j], b, j - i, t)
        R.check_attend(got[i:j], want, {"element": bound, "most": 0.0}, False, b)
        rows -= set(range(i, j))
    if lens[1] > 512:
        rows -= {1, 2}
    assert np.isnan(got[sorted(rows)]).all()


def test_shared_pages_are_given_back_once(dev):
    """Two sequences share their first three pages: the first to end keeps them (keep_len behind them), the last one gives all back."""
    table, free, count = ints([[4, 1, 7, 0, -1], [4, 1, 7, 3, 6]], dev), ints([2, 5, -1, -1, -1, -1, -1, -1], dev), ints([2], dev)
    E.ecco_kv_pages_release(ints([60, 70], dev), ints([60, 48], dev), table, free, count, 16)
    assert int(count) == 4 and free.tolist()[:4] == [2, 5, 3, 6]
    E.ecco_kv_pages_release(ints([60, 48], dev), ints([0, 48], dev), table, free, count, 16)
    assert int(count) == 8 and free.tolist() == [2, 5, 3, 6, 4, 1, 7, 0]


@pytest.mark.parametrize("half", [False, True])
def test_chunks_and_tokens_called_apart(dev, oracle, models, half):
    """A step's chunk and its single tokens in two calls over the same rows, each with its own sequences and bounds: neither touches the other's rows, and each asks for the
    workspace of its own."""
    new, kv, Hq, Hkv = [64] + [1] * 7, [900, 40, 2000, 1, 333, 700, 64, 65], 32, 8
    c = Cache(dev, oracle, models, kv, Hkv, 16, 70)
    q = queries(sum(new), Hq, 71)
    starts, lens, out = ints(np.concatenate([[0], np.cumsum(new)]), dev), ints(kv, dev), torch.full(q.shape, float("nan"), dtype=torch.float16 if half else torch.float32, device=dev)
    qd = torch.from_numpy(q).to(dev)
    for i, j in ((0, 1), (1, 8)):
        size = E.ecco_kv_attend_paged_workspace(sum(new), j - i, Hq, Hkv, max(new[i:j]), max(kv[i:j]), sum(kv[i:j]))
        assert size < 20 * 2 ** 20
        E.ecco_kv_attend_paged(*models, qd, *c.pool, c.table[i:j], starts[i:j + 1], lens[i:j], max(new[i:j]), max(kv[i:j]), sum(kv[i:j]),
                               torch.empty((size,), dtype=torch.uint8, device=dev), out)
        done = int(starts[j])
        assert torch.isfinite(out[:done]).all() and torch.isnan(out[done:]).all()
    got = out.cpu().numpy()
    for b, (n, t) in enumerate(zip(new, kv)):
        at = np.s_[int(starts[b]):int(starts[b + 1])]
        want, bound = c.want(q[at], b, n, t)
        R.check_attend(got[at], want, {"element": bound, "most": float(np.abs(c.values[b].astype(np.float64)).max())}, half, b)
