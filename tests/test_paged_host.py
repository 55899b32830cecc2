"""The paged cache's entry points on a machine without a GPU: what they refuse, in the documented order, before anything is launched; the sizes
of workspaces; and the plain definitions that the GPU tests compare with."""
from __future__ import annotations

import os
import subprocess

import numpy as np
import pytest

import paper_2505_06901_amd as E
from paper_2505_06901_amd import binding, workloads as W

import paged_reference as R

EINVAL, ESHAPE, EALIGN = -1, -2, -3
FAKE, ODD2, ODD4 = 0x1000, 0x1002, 0x1004  # never dereferenced


@pytest.fixture(scope="module")
def model():
    return E.ecco_fit_patterns(W.config_weight("tiny"), 16, 12, 0)


def _call(name, args, **changed):
    a = dict(args)
    assert set(changed) <= set(a), changed
    a.update(changed)
    return getattr(binding.lib(), name)(*a.values())


TAKE = dict(seq_len=FAKE, new_len=FAKE, B=2, page_tokens=16, max_pages=4, page_table=FAKE, free_pages=FAKE, free_count=FAKE, free_left=FAKE, n_pages=8,
            n_tokens=5, q_start=FAKE, kv_len=FAKE, slots=FAKE, stream=None)
RELEASE = dict(seq_len=FAKE, keep_len=FAKE, B=2, page_tokens=16, max_pages=4, page_table=FAKE, free_pages=FAKE, free_count=FAKE, free_left=FAKE, n_pages=8,
               stream=None)
BAD_POOLS = [dict(page_tokens=0), dict(page_tokens=8), dict(page_tokens=24), dict(page_tokens=-16), dict(page_tokens=2048), dict(n_pages=0), dict(n_pages=-1),
             dict(n_pages=1 << 27)]


@pytest.mark.parametrize("name,args", [("ecco_kv_pages_take", TAKE), ("ecco_kv_pages_release", RELEASE)])
def test_pages_refusals(name, args):
    for k, v in args.items():
        if v == FAKE:
            assert _call(name, args, **{k: None}) == EINVAL, k
            assert _call(name, args, **{k: ODD2}) == EALIGN, k
    for bad in BAD_POOLS + [dict(B=0), dict(B=-1), dict(max_pages=0), dict(max_pages=1 << 27)]:
        assert _call(name, args, **bad) == ESHAPE, bad
    if "n_tokens" in args:
        assert _call(name, args, n_tokens=-1) == ESHAPE
        assert _call(name, args, slots=None) == EINVAL
    # in the documented order: null, sizes, alignment
    assert _call(name, args, seq_len=None, B=0) == EINVAL and _call(name, args, seq_len=ODD2, B=0) == ESHAPE


@pytest.mark.parametrize("name", ["ecco_kv_append_paged", "ecco_kv_append_paged_minmax"])
def test_append_refusals(model, name):
    h = model.handle
    args = dict(mk=h, mv=h, k_new=FAKE, v_new=FAKE, k_stride=256, v_stride=256, k_blocks=FAKE, k_meta=FAKE, v_blocks=FAKE, v_meta=FAKE, slots=FAKE, n_tokens=3,
                H=2, n_pages=8, page_tokens=16, stream=None)
    assert _call(name, args) == EINVAL                      # all fine up to the models, which are on no device
    for k in ("mk", "mv", "k_new", "v_new", "k_blocks", "k_meta", "v_blocks", "v_meta", "slots"):
        assert _call(name, args, **{k: None}) == EINVAL, k
    for k in ("k_new", "v_new", "k_meta", "v_meta", "slots"):
        assert _call(name, args, **{k: ODD2}) == EALIGN, k
    for k in ("k_blocks", "v_blocks"):
        assert _call(name, args, **{k: ODD4}) == EALIGN, k
    for bad in BAD_POOLS + [dict(H=0), dict(n_tokens=-1), dict(k_stride=255), dict(k_stride=254), dict(v_stride=257), dict(v_stride=128), dict(k_stride=-256),
                            dict(v_stride=1 << 41), dict(n_tokens=1 << 30, H=4, k_stride=512, v_stride=512)]:
        assert _call(name, args, **bad) == ESHAPE, bad
    assert _call(name, args, n_tokens=0) == EINVAL and _call(name, args, n_tokens=0, mk=None) == EINVAL


ATTEND = dict(mk=0, mv=0, q=FAKE, q_stride=1024, k_blocks=FAKE, k_meta=FAKE, v_blocks=FAKE, v_meta=FAKE, page_table=FAKE, q_start=FAKE, kv_len=FAKE, n_tokens=3,
              B=2, Hq=8, Hkv=2, n_pages=8, page_tokens=16, max_pages=4, max_new=2, max_kv=64, total_kv=100, workspace=FAKE, workspace_bytes=1 << 40, out=FAKE,
              out_half=0, stream=None)


def test_attend_refusals(model):
    args, name = dict(ATTEND, mk=model.handle, mv=model.handle), "ecco_kv_attend_paged"
    assert _call(name, args) == EINVAL                      # the models are on no device
    for k in ("mk", "mv", "q", "k_blocks", "k_meta", "v_blocks", "v_meta", "page_table", "q_start", "kv_len", "out"):
        assert _call(name, args, **{k: None}) == EINVAL, k
    for k in ("k_meta", "v_meta", "page_table", "q_start", "kv_len"):
        assert _call(name, args, **{k: ODD2}) == EALIGN, k
    for k in ("q", "out", "k_blocks", "v_blocks"):
        assert _call(name, args, **{k: ODD4}) == EALIGN, k
    assert _call(name, args, workspace=0x1010) == EALIGN
    assert _call(name, args, out_half=2) == EINVAL and _call(name, args, out_half=-1) == EINVAL
    for bad in BAD_POOLS + [dict(B=0), dict(Hq=0), dict(Hkv=0), dict(Hq=7), dict(Hq=34, q_stride=34 * 128), dict(n_tokens=-1), dict(max_new=0), dict(max_kv=0),
                            dict(total_kv=0), dict(max_pages=0), dict(max_pages=1 << 27), dict(q_stride=1020), dict(q_stride=1016), dict(q_stride=-1024),
                            dict(q_stride=1 << 41), dict(n_tokens=1 << 29)]:
        assert _call(name, args, **bad) == ESHAPE, bad
    assert _call(name, args, B=0, q=ODD4) == ESHAPE and _call(name, args, q=None, B=0) == EINVAL


def test_workspace_sizes():
    need = lambda **c: _call("ecco_kv_attend_paged_workspace", dict(device=-1, n_tokens=8, B=8, Hq=32, Hkv=8, max_new=1, max_kv=4096, total_kv=32768), **c)
    # 64 sequences and heads on 256 compute units: two ranges of tokens for each unit and one more per sequence and head, 8 rows of 130 floats
    assert 0 < need() <= (64 + 512) * 8 * 130 * 4 + 4096
    for none in (dict(n_tokens=0), dict(B=0), dict(Hq=31), dict(Hkv=0), dict(max_new=0), dict(max_kv=0), dict(total_kv=0), dict(n_tokens=-1)):
        assert need(**none) == 0, none
    # more is never enough for less: the sizes grow with the bounds
    for n in (1, 5, 64, 512, 4096):
        assert need(n_tokens=8 * n, max_new=n) <= need(n_tokens=16 * n, max_new=2 * n) + (1 << 30)
    # no sum of sizes runs over
    assert 0 < need(max_kv=(1 << 31) - 1, total_kv=(1 << 34)) < 1 << 50 and need(n_tokens=1 << 24, max_new=1 << 22, max_kv=1 << 22, total_kv=1 << 25) < 1 << 50


def test_reference_take_and_release():
    """The plain definitions on a case worked out by hand: pages of 16, three sequences, five free pages."""
    table = [[7, -1, -1], [3, 4, -1], [-1, -1, -1]]
    t, left, q_start, kv, slots = R.take([10, 32, 0], [7, 1, 3], table, [0, 1, 2, 5, 6, 0, 0, 0], 5, 16, 11)
    assert t.tolist() == [[7, 6, -1], [3, 4, 5], [2, -1, -1]] and left == 2
    assert q_start.tolist() == [0, 7, 8, 11] and kv.tolist() == [17, 33, 3]
    assert slots.tolist() == [7 * 16 + i for i in range(10, 16)] + [96, 80, 32, 33, 34]
    # only one page: the first is served, the second is not, the third needs one as well
    t, left, q_start, kv, slots = R.take([10, 32, 0], [7, 1, 3], table, [6, 0, 0, 0, 0, 0, 0, 0], 1, 16, 11)
    assert kv.tolist() == [17, 0, 0] and left == 0 and (slots[7:] == -1).all()
    free, count = R.release([17, 33, 3], [0, 32, 3], [[7, 6, -1], [3, 4, 5], [2, -1, -1]], [0, 1, 0, 0, 0, 0, 0, 0], 2, 16)
    assert count == 5 and free[:5].tolist() == [0, 1, 7, 6, 5]


def test_reference_attend():
    """A row of a single token is that token's value, a row that sees none is zeros; two equal scores average."""
    v = np.arange(256.0).reshape(2, 128)
    out, bound = R.attend(np.zeros((3, 128)), np.ones((2, 128)), v, np.array([[1, 0], [0, 0], [1, 1]], bool))
    assert np.array_equal(out[0], v[0]) and not out[1].any() and np.allclose(out[2], v.mean(0)) and (bound[1] == 0).all()


@pytest.mark.skipif(not os.path.exists("/opt/rocm/llvm/bin/clang++"), reason="needs ROCm's clang++")
def test_launch_plans_of_rows(tmp_path):
    """tests/plans/rows_plans_main.cpp, compiled with the library's own header, walks the sizes that the kernel is launched with; undefined
    arithmetic is trapped."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    exe = str(tmp_path / "rows_plans")
    cmd = ["/opt/rocm/llvm/bin/clang++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I" + os.path.join(root, "include"),
           "-I" + os.path.join(root, "paper_2505_06901_amd", "csrc"), os.path.join(root, "tests", "plans", "rows_plans_main.cpp"), "-o", exe]
    build = subprocess.run(cmd, capture_output=True, text=True)
    assert build.returncode == 0, build.stderr[-4000:]
    run = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and "conditions hold" in run.stdout, (run.stdout[-2000:], run.stderr[-2000:])


def test_ranges_fit_what_the_launch_holds(tmp_path):
    """tests/plans/range_plans_main.cpp: sequences so long that their units together exceed an int included; undefined arithmetic is trapped."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    exe = str(tmp_path / "range_plans")
    cmd = ["/opt/rocm/llvm/bin/clang++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I" + os.path.join(root, "include"),
           "-I" + os.path.join(root, "paper_2505_06901_amd", "csrc"), os.path.join(root, "tests", "plans", "range_plans_main.cpp"), "-o", exe]
    build = subprocess.run(cmd, capture_output=True, text=True)
    assert build.returncode == 0, build.stderr[-4000:]
    run = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and "conditions hold" in run.stdout, (run.stdout[-2000:], run.stderr[-2000:])


@pytest.mark.parametrize("other", ["seq_len", "new_len"])
def test_lengths_are_not_advanced_in_place(other):
    """kv_len is written by one workgroup while others read the lengths, so it cannot be one of them: refused behind all other checks."""
    apart = {k: FAKE + 0x100 * i for i, k in enumerate(TAKE) if TAKE[k] == FAKE}
    same = {**apart, "kv_len": apart[other]}
    assert _call("ecco_kv_pages_take", TAKE, **same) == EINVAL
    assert _call("ecco_kv_pages_take", TAKE, **{**same, "B": 0}) == ESHAPE
    assert _call("ecco_kv_pages_take", TAKE, **{**same, "slots": ODD2}) == EALIGN
