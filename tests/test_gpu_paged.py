"""The paged compressed cache on the GPU: pages taken and given back, chunks appended by slot, attention of new tokens over pages, against the
plain definitions (paged_reference.py, 64 bits) and the oracle's encoder and decoder; and all of them together, as a server uses them."""
from __future__ import annotations

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2505_06901_amd as E  # noqa: E402
from paper_2505_06901_amd import workloads as W  # noqa: E402

import paged_reference as R  # noqa: E402
from test_gpu_parity import _skewed_data, _skewed_model  # noqa: E402


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


def ints(a, dev):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(dev)


def host(t):
    return t.cpu().numpy()


# ---- pages ----------------------------------------------------------------------------------------------------------
def _lists(rng, B, page, most, spare):
    """Lengths, a table of pages in random order, and a stack of what is left."""
    held = rng.integers(0, most + 1, B)
    n = -(-held // page)
    n_pages = int(n.sum()) + spare
    order = rng.permutation(n_pages)
    max_pages = -(-most // page) + 3
    table, at = np.full((B, max_pages), -1), 0
    for b in range(B):
        table[b, :n[b]] = order[at:at + n[b]]
        at += n[b]
    free = np.full(n_pages, -7)
    free[:spare] = order[at:]
    return held, table, free, spare


@pytest.mark.parametrize("B,page,most,new,spare", [
    (1, 16, 0, 1, 1), (1, 16, 15, 1, 4), (7, 16, 100, 40, 30), (64, 32, 500, 1, 64), (257, 16, 300, 3, 200),   # in the last ones pages run out
    (1024, 16, 40, 1, 500), (1025, 64, 200, 5, 1025), (2100, 16, 64, 2, 700), (3, 1024, 5000, 3000, 12), (40, 16, 64, 200, 600),
])
@pytest.mark.parametrize("seed", [0, 1])
def test_take(dev, B, page, most, new, spare, seed):
    rng = np.random.default_rng(seed + 17 * B)
    held, table, free, count = _lists(rng, B, page, most, spare)
    fresh = rng.integers(0, new + 1, B)
    if seed:  # negative lengths are none; an entry that is no page gives no slots
        held[rng.integers(0, B)], fresh[rng.integers(0, B)] = -5, -9
        table[rng.integers(0, B), 0] = [-1, len(free), 2 ** 31 - 1, -2 ** 31][B % 4]
        if B > 2:  # more than the table holds
            fresh[B // 2] = 2 ** 31 - 1 if B % 2 else (table.shape[1] + 1) * page
    rows = int(np.minimum(np.maximum(fresh, 0), 10 ** 6).sum())
    for n_tokens in sorted({rows, rows + 5, rows - min(rows, 3), 0} if rows < 200000 else {5000}):
        want = R.take(held, fresh, table, free, count, page, n_tokens)
        t, c = ints(table, dev), ints([count], dev)
        slots = torch.full((n_tokens + 1,), -99, dtype=torch.int32, device=dev)
        q_start, kv_len, _ = E.ecco_kv_pages_take(ints(held, dev), ints(fresh, dev), t, ints(free, dev), c, page, n_tokens, slots=slots)
        assert np.array_equal(host(t), want[0]) and int(c) == want[1], n_tokens
        assert np.array_equal(host(q_start), want[2]) and np.array_equal(host(kv_len), want[3]), n_tokens
        assert np.array_equal(host(slots)[:-1], want[4]) and int(slots[-1]) == -99, n_tokens


@pytest.mark.parametrize("B,page,most,new,spare", [(300, 16, 200, 60, 900), (1500, 16, 40, 9, 3000), (2, 1024, 9000, 30000, 80)])
def test_take_with_a_count_of_its_own(dev, B, page, most, new, spare):
    """Many rows: the same result whether the count is updated in place or written elsewhere, several times over."""
    rng = np.random.default_rng(B)
    held, table, free, count = _lists(rng, B, page, most, spare)
    fresh = rng.integers(0, new + 1, B)
    table = np.concatenate([table, np.full((B, -(-new // page)), -1)], 1)
    n_tokens = int(fresh.sum())
    want = R.take(held, fresh, table, free, count, page, n_tokens)
    for i in range(4):
        t, c, left = ints(table, dev), ints([count], dev), ints([-1], dev)
        q_start, kv_len, slots = E.ecco_kv_pages_take(ints(held, dev), ints(fresh, dev), t, ints(free, dev), c, page, n_tokens, free_left=left if i % 2 else None)
        assert int(left if i % 2 else c) == want[1] and (i % 2 == 0 or int(c) == count)
        for got, w in zip((t, q_start, kv_len, slots), (want[0], *want[2:])):
            assert np.array_equal(host(got), w)


@pytest.mark.parametrize("count", [-3, 0, 5, 100])
def test_take_reads_the_count_as_what_the_stack_can_hold(dev, count):
    held, fresh, table, free = [3, 0, 0], [20, 16, 16], np.full((3, 4), 0), np.arange(8)[::-1].copy()
    want = R.take(held, fresh, table, free, count, 16, 52)
    t, c, left = ints(table, dev), ints([count], dev), ints([-1], dev)
    q_start, kv_len, slots = E.ecco_kv_pages_take(ints(held, dev), ints(fresh, dev), t, ints(free, dev), c, 16, 52, free_left=left)
    assert int(c) == count and int(left) == want[1]
    assert np.array_equal(host(t), want[0]) and np.array_equal(host(slots), want[4]) and np.array_equal(host(kv_len), want[3])


@pytest.mark.parametrize("B,page,most,spare", [(1, 16, 50, 1), (5, 16, 200, 7), (300, 16, 4000, 10), (1030, 32, 300, 0), (2500, 16, 90, 3)])
def test_release(dev, B, page, most, spare):
    rng = np.random.default_rng(B)
    held, table, free, count = _lists(rng, B, page, most, spare)
    keep = np.where(rng.random(B) < 0.4, 0, np.where(rng.random(B) < 0.5, held, held - rng.integers(0, 40, B)))
    table[rng.integers(0, B, max(1, B // 10)), 0] = [-1, len(free), 2 ** 31 - 1, -2 ** 31][B % 4]  # no pages: left out
    before = ints(table, dev)
    want = R.release(held, keep, table, free, count, page)
    f, c, left = ints(free, dev), ints([count], dev), ints([0], dev)
    E.ecco_kv_pages_release(ints(held, dev), ints(keep, dev), before, f, c, page, free_left=left)
    assert int(left) == want[1] and int(c) == count and np.array_equal(host(f), want[0]) and np.array_equal(host(before), table)
    E.ecco_kv_pages_release(ints(held, dev), ints(keep, dev), before, f, c, page)  # in place, onto the same count
    assert int(c) == want[1] and np.array_equal(host(f), want[0])
    # a second time on top: what exceeds the stack is dropped
    again = R.release(held, keep, table, want[0], want[1], page)
    E.ecco_kv_pages_release(ints(held, dev), ints(keep, dev), before, f, c, page)
    assert int(c) == again[1] <= len(free) and np.array_equal(host(f), again[0])


def test_release_what_was_taken(dev):
    rng = np.random.default_rng(5)
    held, table, free, count = _lists(rng, 50, 16, 300, 400)
    fresh = rng.integers(0, 90, 50)
    t, f, c = ints(table, dev), ints(free, dev), ints([count], dev)
    _, kv_len, _ = E.ecco_kv_pages_take(ints(held, dev), ints(fresh, dev), t, f, c, 16, int(fresh.sum()))
    assert int(c) < count and np.array_equal(host(kv_len), held + fresh)
    E.ecco_kv_pages_release(kv_len, ints(held, dev), t, f, c, 16)
    assert int(c) == count and sorted(host(f)[:count].tolist()) == sorted(free[:count].tolist())


# ---- append ---------------------------------------------------------------------------------------------------------
@pytest.fixture(scope="module")
def models(dev, oracle):
    """(K, V) models by name: 16 and 64 patterns, one pattern, and codes of up to 12 bits."""
    k, v = W.kv_cache(1, 4, 192, 128, seed=3)
    made = {s: tuple(E.ecco_model_to_device(E.ecco_fit_patterns(x, s, 12, 5), 0) for x in (k, v)) for s in (1, 16, 64)}
    cent, lens, probs = _skewed_model(oracle, 8, 21)
    made["long"] = (E.ecco_model_to_device(E.ecco_model_create(cent, lens), 0),) * 2
    made["long values"] = (made[16][0], made["long"][1])
    made["long keys"] = (made["long"][0], made[64][1])
    made["probs"] = (cent, probs)
    return made


def _values(models, which, rows, H, seed):
    """Keys and values [rows, H, 128] FP16 that suit the models."""
    k, v = W.kv_cache(1, H, rows, 128, seed=seed)
    k, v = (np.ascontiguousarray(x[0].transpose(1, 0, 2)) for x in (k, v))
    skewed = lambda s: _skewed_data(*models["probs"], rows * H, s).reshape(rows, H, 128).view(np.float16)
    if which in ("long", "long keys"):
        k = skewed(seed + 1)
    if which in ("long", "long values"):
        v = skewed(seed + 2)
    return k, v


def _encode(oracle, m, x, minmax=False):
    f = oracle.encode_minmax if minmax else oracle.encode
    return f(m.centroids, m.code_lens, np.ascontiguousarray(x).reshape(-1, 128).view(np.uint16))


@pytest.mark.parametrize("minmax", [False, True])
@pytest.mark.parametrize("which,rows,H,page,fused", [
    (16, 1, 1, 16, False), (64, 3, 5, 32, True), (16, 130, 4, 16, True), (64, 700, 4, 128, True), (1, 90, 3, 64, False), ("long", 60, 2, 16, True),
    ("long values", 1000, 3, 1024, True), (64, 900, 4, 16, False), ("long", 1200, 3, 32, False),
])
def test_append(dev, oracle, models, minmax, which, rows, H, page, fused):
    mk, mv = models[which]
    k, v = _values(models, which, rows, H, 40 + rows)
    if rows > 5:
        k[5] = 0
        v[4, 0] = k[5, 0]
    rng = np.random.default_rng(rows)
    n_pages = -(-rows // page) + 3
    slots = rng.permutation(n_pages * page)[:rows]
    if rows > 2:  # rows that have no slot
        slots[[0, rows // 2, rows - 1]] = [-1, n_pages * page, -2 ** 31]
    pools, want = [], []
    for x, m in ((k, mk), (v, mv)):
        blocks, meta = rng.integers(0, 256, (n_pages, H, page, 64), np.uint8), rng.integers(0, 2 ** 31, (n_pages, H, page), np.int32)
        pools += [torch.from_numpy(blocks).to(dev), torch.from_numpy(meta).to(dev)]
        ob, om = _encode(oracle, m, x, minmax)
        ob, om = ob.reshape(rows, H, 64), om.view(np.int32).reshape(rows, H)
        for i, s in enumerate(slots):
            if 0 <= s < n_pages * page:
                blocks[s // page, :, s % page], meta[s // page, :, s % page] = ob[i], om[i]
        want += [blocks, meta]
    if fused:  # rows of a wider tensor, the keys two heads in
        wide = torch.full((rows, 2 * H + 3, 128), float("nan"), dtype=torch.float16, device=dev)
        wide[:, 2:2 + H], wide[:, 2 + H:2 + 2 * H] = torch.from_numpy(k).to(dev), torch.from_numpy(v).to(dev)
        kt, vt = wide[:, 2:2 + H], wide[:, 2 + H:2 + 2 * H]
    else:
        kt, vt = torch.from_numpy(k).to(dev), torch.from_numpy(v).to(dev)
    call = E.ecco_kv_append_paged_minmax if minmax else E.ecco_kv_append_paged
    call(mk, mv, kt, vt, pools[0], pools[1], pools[2], pools[3], ints(slots, dev))
    for got, w in zip(pools, want):
        assert np.array_equal(host(got), w)
    call(mk, mv, kt[:0], vt[:0], pools[0], pools[1], pools[2], pools[3], ints(slots, dev))  # nothing to do
    for got, w in zip(pools, want):
        assert np.array_equal(host(got), w)


# ---- attention ------------------------------------------------------------------------------------------------------
class Cache:
    """A pool filled by the oracle's encoder, pages in random order, unused slots and pages full of ones (NaN scales)."""

    def __init__(self, dev, oracle, models, which, lens, Hkv, page, seed, holes=()):
        rng = np.random.default_rng(seed)
        self.Hkv, self.page, self.lens = Hkv, page, list(lens)
        n = [-(-t // page) for t in lens]
        n_pages = sum(n) + 2
        order, at = rng.permutation(n_pages), 0
        max_pages = max(n + [1]) + 2
        self.table = np.full((len(lens), max_pages), 2 ** 31 - 1)
        mk, mv = self.models = models[which]
        self.keys, self.values, pool = [], [], [np.full((n_pages, Hkv, page, 64), 255, np.uint8), np.full((n_pages, Hkv, page), -1, np.int32),
                                                np.full((n_pages, Hkv, page, 64), 255, np.uint8), np.full((n_pages, Hkv, page), -1, np.int32)]
        for b, t in enumerate(lens):
            self.table[b, :n[b]] = order[at:at + n[b]]
            at += n[b]
            if t == 0:
                self.keys.append(np.zeros((0, Hkv, 128), np.float16))
                self.values.append(np.zeros((0, Hkv, 128), np.float16))
                continue
            pages, off = np.repeat(self.table[b, :n[b]], page)[:t], np.tile(np.arange(page), n[b])[:t]
            for i, (x, m, kept) in enumerate(zip(_values(models, which, t, Hkv, seed + 100 * b), (mk, mv), (self.keys, self.values))):
                blocks, meta = _encode(oracle, m, x)
                pool[2 * i][pages, :, off], pool[2 * i + 1][pages, :, off] = blocks.reshape(t, Hkv, 64), meta.view(np.int32).reshape(t, Hkv)
                kept.append(oracle.decode(m.centroids, m.code_lens, blocks, meta).view(np.float16).reshape(t, Hkv, 128))
        for b, i, what in holes:
            self.table[b, i] = what
        self.n_pages = n_pages
        self.pool = [torch.from_numpy(a).to(dev) for a in pool]

    def want(self, q, new, kv):
        """(outputs, bounds) of all rows, [rows, Hq, 128]."""
        out, element, most, row = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape), 0
        grp = q.shape[1] // self.Hkv
        for b, (n, t) in enumerate(zip(new, kv)):
            real = (self.table[b, np.arange(t) // self.page] >= 0) & (self.table[b, np.arange(t) // self.page] < self.n_pages)
            seen = (np.arange(t)[None, :] <= (t - n + np.arange(n))[:, None]) & real
            for h in range(self.Hkv):
                k, v = self.keys[b][:t, h], self.values[b][:t, h]
                rows = q[row:row + n, h * grp:(h + 1) * grp].reshape(n * grp, 128)
                o, e = R.attend(rows, k, v, np.repeat(seen, grp, 0))
                at = np.s_[row:row + n, h * grp:(h + 1) * grp]
                out[at], element[at] = o.reshape(n, grp, 128), e.reshape(n, grp, 128)
                most[at] = np.abs(v.astype(np.float64)).max(0, initial=0.0)
            row += n
        return out, {"element": element, "most": most}

    def run(self, dev, q, new, kv, half, pad=0, max_new=None, max_kv=None, total_kv=None, **kw):
        starts = np.concatenate([[0], np.cumsum(new)])
        n = int(starts[-1])
        out = torch.full((n + pad, q.shape[1], 128), float("nan"), dtype=torch.float16 if half else torch.float32, device=dev)
        wide = torch.full((n + pad, q.shape[1] + 3, 128), float("nan"), dtype=torch.float16, device=dev)  # rows behind the last are NaN
        wide[:n, 1:-2] = torch.from_numpy(q).to(dev)
        E.ecco_kv_attend_paged(*self.models, wide[:, 1:-2], *self.pool, ints(self.table, dev), ints(starts, dev), ints(kv, dev),
                               max_new or max(max(new), 1), max_kv or max(max(kv), 1), total_kv or max(sum(kv), 1), out=out, **kw)
        assert torch.isnan(out[n:]).all()  # left as they were
        return host(out[:n])


def _queries(rows, Hq, seed):
    return W.activation(rows * Hq, 128, seed).reshape(rows, Hq, 128)


ATTEND = [
    # which, Hq, Hkv, page, [(new, kv)]
    (16, 1, 1, 16, [(1, 1)]),
    (16, 4, 1, 16, [(1, 31)]),
    (64, 4, 4, 32, [(1, 33), (1, 0), (0, 40), (1, 64)]),              # a sequence without tokens, one without rows
    (16, 8, 2, 16, [(1, 500), (1, 17), (1, 1), (1, 256)]),
    (64, 32, 2, 64, [(1, 300), (1, 129)]),                             # groups of 16
    (16, 18, 2, 32, [(2, 300), (1, 200)]),                             # groups of 9: 18 rows
    (16, 8, 2, 16, [(5, 300), (3, 3), (4, 2), (7, 1), (2, 0)]),        # rows before position 0, sequences shorter than their rows
    ("long", 8, 2, 16, [(1, 200), (3, 99)]),
    ("long values", 6, 2, 128, [(1, 400), (2, 100)]),
    ("long keys", 4, 4, 16, [(4, 250)]),
    (1, 2, 1, 1024, [(1, 1500), (2, 1025)]),
    (64, 4, 1, 16, [(1, 5000)]),                                       # split over the tokens
    (16, 2, 2, 32, [(1, 9000), (1, 40)]),
    (16, 4, 2, 16, [(1, 40)] * 300),                                   # more sequences and heads than compute units
    (16, 8, 2, 16, [(40, 40)]),                                        # a prompt
    (64, 8, 2, 32, [(33, 100), (1, 70), (64, 64), (9, 200)]),          # chunks beside sequences that decode
    (16, 4, 1, 16, [(130, 417), (127, 127), (1, 417)]),
    (16, 3, 3, 64, [(129, 600), (50, 333)]),                           # a cache per query head
    (16, 32, 2, 16, [(17, 90), (5, 1000)]),
    ("long", 8, 2, 16, [(70, 300)]),
    (64, 16, 2, 128, [(100, 20), (60, 59), (90, 0)]),                  # chunks of which much comes before position 0
    (16, 8, 1, 16, [(300, 1200)]),
    (16, 4, 1, 16, [(1, 30 + 17 * i % 500) for i in range(100)]),      # ranges over more sequences than a wavefront has lanes
    (16, 2, 1, 32, [(40 if i % 9 == 4 else 1 + i % 2, 60 + 31 * i % 200) for i in range(70)]),  # chunks among as many
    (64, 128, 8, 64, [(790, 800)]),                                    # tiles of 256 rows
    (16, 32, 4, 16, [(11, 3000), (2, 1100), (160, 2048)]),             # 8 rows per token: few, and tiles split over the tokens
]


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("case", range(len(ATTEND)))
def test_attend(dev, oracle, models, case, half):
    which, Hq, Hkv, page, spans = ATTEND[case]
    new, kv = [n for n, _ in spans], [t for _, t in spans]
    c = Cache(dev, oracle, models, which, kv, Hkv, page, 7 + case)
    q = _queries(sum(new), Hq, 300 + case)
    want, bound = c.want(q, new, kv)
    R.check_attend(c.run(dev, q, new, kv, half, pad=case % 3), want, bound, half, ATTEND[case])
    # larger bounds than needed: other launches, the same result
    got = c.run(dev, q, new, kv, half, max_new=max(new) + 40, max_kv=2 * max(max(kv), 1) + 100, total_kv=3 * sum(kv) + 1000)
    R.check_attend(got, want, bound, half, ATTEND[case])


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("page,spans,holes", [
    (16, [(1, 200), (3, 90)], [(0, 0, -1), (0, 5, 10 ** 6), (1, 2, -2 ** 31)]),
    (32, [(1, 200), (60, 90)], [(0, 6, -1), (1, 0, 2 ** 31 - 1)]),       # the last page, the first page
    (16, [(90, 90)], [(0, 0, -1), (0, 3, -5)]),                          # the first rows see nothing
    (64, [(1, 60), (50, 50)], [(0, 0, -1), (1, 0, -1)]),                 # no page at all
])
def test_attend_without_some_pages(dev, oracle, models, page, spans, holes, half):
    new, kv = [n for n, _ in spans], [t for _, t in spans]
    c = Cache(dev, oracle, models, 16, kv, 2, page, 90, holes)
    q = _queries(sum(new), 8, 91)
    want, bound = c.want(q, new, kv)
    R.check_attend(c.run(dev, q, new, kv, half), want, bound, half)


def test_attend_lengths_beyond_the_bounds_touch_nothing_else(dev, oracle, models):
    """Lengths on the device that the host's bounds do not cover, and starts that do not ascend: rows may be left unwritten, other sequences' rows
    within the bounds and rows behind the last are what they are."""
    spans = [(1, 300), (2, 500), (1, 100)]
    new, kv = [n for n, _ in spans], [t for _, t in spans]
    c = Cache(dev, oracle, models, 16, kv, 2, 16, 60)
    q = _queries(4, 8, 61)
    want, _ = c.want(q, new, kv)
    guard = torch.full((6, 8, 128), float("nan"), dtype=torch.float32, device=dev)
    qd = torch.from_numpy(np.concatenate([q, q[:2]])).to(dev)
    for starts, lens in (([0, 1, 3, 4], [300, 2 ** 31 - 1, 100]), ([0, 1, 3, 2 ** 31 - 1], [300, 500, -4]), ([0, 1, -7, 1], [300, 500, 100])):
        E.ecco_kv_attend_paged(*c.models, qd[:4], *c.pool, ints(c.table, dev), ints(starts, dev), ints(lens, dev), 2, 512, 900, out=guard[:4])
        torch.cuda.synchronize()
        assert torch.isnan(guard[4:]).all()
        assert np.abs(host(guard[0]) - want[0]).max() <= 1e-3


def test_attend_sequences_that_share_pages(dev, oracle, models):
    """Two sequences with the same pages in front, and one that reads the same page twice."""
    c = Cache(dev, oracle, models, 16, [150, 150, 64], 2, 32, 95)
    c.table[1, :3] = c.table[0, :3]
    c.table[2, 1] = c.table[2, 0]
    for kept in (c.keys, c.values):
        kept[1][:96] = kept[0][:96]
        kept[2][32:] = kept[2][:32]
    new, kv = [2, 60, 1], [150, 150, 64]
    q = _queries(63, 8, 96)
    want, bound = c.want(q, new, kv)
    R.check_attend(c.run(dev, q, new, kv, False), want, bound, False)


def test_attend_beyond_4_gib(dev, oracle, models):
    """A pool whose blocks and meta words lie beyond offsets of 32 bits."""
    Hkv, page, n_pages = 8, 1024, 9000  # 4.4 GiB of blocks each for keys and values
    new, kv = [1, 60, 3], [1500, 100, 700]
    c = Cache(dev, oracle, models, 16, kv, Hkv, page, 70)
    pool = [torch.empty((n_pages, *a.shape[1:]), dtype=a.dtype, device=dev) for a in c.pool]
    moved = {p: n_pages - 1 - 3 * i if i % 2 else 8300 + i for i, p in enumerate(range(c.n_pages))}
    for p, to in moved.items():
        for big, small in zip(pool, c.pool):
            big[to] = small[p]
    q = _queries(sum(new), 16, 71)
    want, bound = c.want(q, new, kv)
    c.table = np.vectorize(lambda p: moved.get(p, -1))(c.table)
    c.pool = pool
    R.check_attend(c.run(dev, q, new, kv, False), want, bound, False)
    # and the append there
    k, v = _values(models, 16, 5, Hkv, 72)
    slots = [(n_pages - 2) * page + 3, 8600 * page, 8600 * page + 1, 1, (n_pages - 1) * page + page - 1 if n_pages - 1 not in moved.values() else 8600 * page + 2]
    E.ecco_kv_append_paged(*c.models, torch.from_numpy(k).to(dev), torch.from_numpy(v).to(dev), *pool, ints(slots, dev))
    for x, m, blocks, meta in ((k, c.models[0], pool[0], pool[1]), (v, c.models[1], pool[2], pool[3])):
        ob, om = _encode(oracle, m, x)
        for i, s in enumerate(slots):
            assert np.array_equal(host(blocks[s // page, :, s % page]), ob.reshape(5, Hkv, 64)[i])
            assert np.array_equal(host(meta[s // page, :, s % page]).view(np.uint32), om.reshape(5, Hkv)[i])


# ---- together -------------------------------------------------------------------------------------------------------
class Server:
    """A paged cache as a program keeps it: chunks of prompts, then steps of one token, all lengths on the device."""

    def __init__(self, dev, models, which, B, Hq, Hkv, page, n_pages, max_pages, seed):
        self.dev, self.m, self.B, self.Hq, self.Hkv, self.page, self.max_pages = dev, models[which], B, Hq, Hkv, page, max_pages
        rng = np.random.default_rng(seed)
        self.table, self.free = ints(np.full((B, max_pages), -1), dev), ints(rng.permutation(n_pages), dev)
        self.count, self.lens = ints([n_pages], dev), ints(np.zeros(B), dev)
        self.pool = [torch.zeros((n_pages, Hkv, page, 64), dtype=torch.uint8, device=dev), torch.zeros((n_pages, Hkv, page), dtype=torch.int32, device=dev),
                     torch.zeros((n_pages, Hkv, page, 64), dtype=torch.uint8, device=dev), torch.zeros((n_pages, Hkv, page), dtype=torch.int32, device=dev)]
        self.held = [np.zeros((2, 0, Hkv, 128), np.float16) for _ in range(B)]

    def step(self, new, qkv, max_new, max_kv, out=None, workspace=None):
        """qkv [rows, Hq + 2 Hkv, 128] on the device; new: int32 tensor.  Lengths advance on the device."""
        Hq, Hkv = self.Hq, self.Hkv
        q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        q_start, kv_len, slots = E.ecco_kv_pages_take(self.lens, new, self.table, self.free, self.count, self.page, qkv.shape[0])
        E.ecco_kv_append_paged(*self.m, k, v, *self.pool, slots)
        out = E.ecco_kv_attend_paged(*self.m, q, *self.pool, self.table, q_start, kv_len, max_new, max_kv, out=out, workspace=workspace)
        self.lens.copy_(kv_len)
        return out


def test_server_steps_match_the_contiguous_cache(dev, oracle, models):
    """Chunked prompts, decoding, drafted tokens taken back, a request that ends and one that takes its pages: against 64 bits at every step, and the
    decoding steps against the library's contiguous cache, which holds the same blocks."""
    B, Hq, Hkv, page, n_pages, max_pages = 3, 8, 2, 16, 40, 24
    s = Server(dev, models, 16, B, Hq, Hkv, page, n_pages, max_pages, 3)
    mk, mv = s.m
    T_max, keys, values = max_pages * page, [np.zeros((0, Hkv, 128), np.float16)] * B, [np.zeros((0, Hkv, 128), np.float16)] * B
    flat = [torch.zeros((B, Hkv, T_max, 64), dtype=torch.uint8, device=dev), torch.zeros((B, Hkv, T_max), dtype=torch.int32, device=dev),
            torch.zeros((B, Hkv, T_max, 64), dtype=torch.uint8, device=dev), torch.zeros((B, Hkv, T_max), dtype=torch.int32, device=dev)]
    decoded = lambda m, x: oracle.decode(m.centroids, m.code_lens, *_encode(oracle, m, x)).view(np.float16).reshape(x.shape)
    plan = [[100, 30, 0], [57, 1, 70], [1, 1, 1], [1, 1, 1], [4, 4, 4], "back", [1, 1, 1], "done", [90, 1, 1], [1, 1, 1]]
    for i, new in enumerate(plan):
        if isinstance(new, str):
            lens = host(s.lens)
            keep = np.array([len(k) for k in keys]) - (3 if new == "back" else 0)
            if new == "done":
                keep[0] = 0
            E.ecco_kv_pages_release(s.lens, ints(keep, dev), s.table, s.free, s.count, page)
            assert int(s.count) == n_pages - sum(-(-k // page) for k in keep.tolist()) and (lens >= keep).all()
            s.lens.copy_(ints(keep, dev))
            keys, values = [k[:n] for k, n in zip(keys, keep)], [v[:n] for v, n in zip(values, keep)]
            continue
        rows = sum(new)
        q = _queries(rows, Hq, 500 + i)
        k, v = _values(models, 16, rows, Hkv, 600 + i)
        qkv = torch.from_numpy(np.concatenate([q, k, v], 1)).to(dev)
        got = host(s.step(ints(new, dev), qkv, max(new), 400))
        row = 0
        held = [len(x) for x in keys]
        for b, n in enumerate(new):
            keys[b], values[b] = (np.concatenate([old, decoded(m, x[row:row + n])]) if n else old for old, x, m in ((keys[b], k, mk), (values[b], v, mv)))
            t = len(keys[b])
            seen = np.repeat(np.arange(t)[None, :] <= (t - n + np.arange(n))[:, None], Hq // Hkv, 0)
            for h in range(Hkv):
                at = np.s_[row:row + n, h * 4:(h + 1) * 4]
                o, e = R.attend(q[at].reshape(-1, 128), keys[b][:, h], values[b][:, h], seen)
                R.check_attend(got[at].reshape(-1, 128), o, {"element": e, "most": 0.0}, False, (i, b, h))
            row += n
        assert np.array_equal(host(s.lens), [len(x) for x in keys])
        # the contiguous cache: one token after the other
        for j in range(max(new)):
            starts = np.cumsum([0] + new)
            pick = [starts[b] + min(j, max(n - 1, 0)) if n else 0 for b, n in enumerate(new)]
            at = ints([held[b] + j if j < n else -1 for b, n in enumerate(new)], dev)
            E.ecco_kv_append(mk, mv, qkv[pick, Hq:Hq + Hkv].contiguous(), qkv[pick, Hq + Hkv:].contiguous(), *flat, at, B, Hkv, T_max)
        if new == [1, 1, 1]:
            ref = E.ecco_kv_attend_gqa(mk, mv, qkv[:, :Hq].contiguous(), *flat, s.lens, B, Hq, Hkv, T_max)
            assert np.abs(got - host(ref)).max() <= 1e-4 * np.abs(host(ref)).max()


def test_captured_step_replays(dev, oracle, models):
    """A whole step in a graph, lengths advancing on the device, with eager work between the replays; every replay against an eager twin."""
    B, Hq, Hkv, page = 4, 8, 2, 16
    servers = [Server(dev, models, 16, B, Hq, Hkv, page, 60, 12, 3) for _ in range(2)]
    prompt = torch.from_numpy(np.concatenate([_queries(100, Hq, 1), *_values(models, 16, 100, Hkv, 2)], 1)).to(dev)
    first = ints([40, 20, 39, 1], dev)
    for s in servers:
        s.step(first, prompt, 40, 100)
    one, qkv = ints([1, 1, 1, 1], dev), torch.zeros((B, Hq + 2 * Hkv, 128), dtype=torch.float16, device=dev)
    a, b = servers
    out = torch.zeros((B, Hq, 128), dtype=torch.float32, device=dev)
    size = E.ecco_kv_attend_paged_workspace(B, B, Hq, Hkv, 1, 192, B * 192)
    ws = torch.empty((max(size, 1),), dtype=torch.uint8, device=dev)
    kept = [t.clone() for t in (a.table, a.count, a.lens)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a.step(one, qkv, 1, 192, out=out, workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    for t, old in zip((a.table, a.count, a.lens), kept):
        t.copy_(old)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.step(one, qkv, 1, 192, out=out, workspace=ws)
    for i in range(20):  # over the borders of pages
        fresh = torch.from_numpy(np.concatenate([_queries(B, Hq, 10 + i), *_values(models, 16, B, Hkv, 30 + i)], 1)).to(dev)
        qkv.copy_(fresh)
        graph.replay()
        want = b.step(one, fresh, 1, 192)
        torch.cuda.synchronize()
        assert torch.equal(out, want), i
        for x, y in ((a.table, b.table), (a.count, b.count), (a.lens, b.lens), (a.pool[1], b.pool[1]), (a.pool[2], b.pool[2])):
            assert torch.equal(x, y), i


def test_captured_chunks_replay_with_other_lengths(dev, oracle, models):
    """Chunks beside single tokens in a graph: the lengths, tables and queries of every replay are others, with eager work in between."""
    Hq, Hkv, page, lens = 8, 2, 16, [700, 500, 260, 90]
    c = Cache(dev, oracle, models, 16, lens, Hkv, page, 97)
    n_tokens, max_new, max_kv, total = 200, 150, 700, 1600
    q = torch.zeros((n_tokens, Hq, 128), dtype=torch.float16, device=dev)
    starts, kv, out = ints(np.zeros(5), dev), ints(np.zeros(4), dev), torch.zeros((n_tokens, Hq, 128), dtype=torch.float32, device=dev)
    ws = torch.empty((E.ecco_kv_attend_paged_workspace(n_tokens, 4, Hq, Hkv, max_new, max_kv, total),), dtype=torch.uint8, device=dev)
    table = ints(c.table, dev)
    call = lambda o, w: E.ecco_kv_attend_paged(*c.models, q, *c.pool, table, starts, kv, max_new, max_kv, total, w, o)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(out, ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out, ws)
    rng = np.random.default_rng(3)
    for i in range(6):
        new = [[150, 1, 1, 1], [1, 1, 1, 1], [1, 90, 0, 40], [0, 0, 100, 1], [5, 33, 130, 32], [1, 1, 3, 2]][i]
        now = [int(rng.integers(max(n, 1), t + 1)) for n, t in zip(new, lens)]
        qh = _queries(n_tokens, Hq, 700 + i)
        q.copy_(torch.from_numpy(qh))
        starts.copy_(ints(np.concatenate([[0], np.cumsum(new)]), dev))
        kv.copy_(ints(now, dev))
        out.fill_(-3.0)
        graph.replay()
        eager = call(torch.full_like(out, -3.0), None)
        assert torch.equal(out, eager), i
        rows = sum(new)
        want, bound = c.want(qh[:rows], new, now)
        R.check_attend(host(out)[:rows], want, bound, False, i)
        assert bool((out[rows:] == -3.0).all())


def test_streams_and_repeatability(dev, oracle, models):
    """The same call on two streams at once, each with its workspace, several times over: the same bits."""
    new, kv = [1, 70, 5], [900, 600, 333]
    c = Cache(dev, oracle, models, 64, kv, 2, 16, 80)
    q = torch.from_numpy(_queries(sum(new), 8, 81)).to(dev)
    args = (*c.models, q, *c.pool, ints(c.table, dev), ints(np.concatenate([[0], np.cumsum(new)]), dev), ints(kv, dev), 70, 900, 1833)
    first = E.ecco_kv_attend_paged(*args)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for _ in range(5):
        for st in streams:
            with torch.cuda.stream(st):
                outs.append(E.ecco_kv_attend_paged(*args))
    torch.cuda.synchronize()
    assert all(torch.equal(o, first) for o in outs)


def test_attend_refuses_a_workspace_that_is_too_small(dev, oracle, models):
    new, kv = [1, 70], [3000, 600]
    c = Cache(dev, oracle, models, 16, kv, 1, 16, 85)
    q = torch.from_numpy(_queries(71, 4, 86)).to(dev)
    size = E.ecco_kv_attend_paged_workspace(71, 2, 4, 1, 70, 3000, 3600)
    assert size > 0
    for ws in (torch.empty((size - 1,), dtype=torch.uint8, device=dev), torch.empty((0,), dtype=torch.uint8, device=dev)):
        with pytest.raises(E.EccoError) as e:
            E.ecco_kv_attend_paged(*c.models, q, *c.pool, ints(c.table, dev), ints([0, 1, 71], dev), ints(kv, dev), 70, 3000, 3600, workspace=ws)
        assert e.value.status == -1
