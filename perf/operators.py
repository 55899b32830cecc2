"""The operators of the paged compressed cache, in their plain form and through the library's entry points.

A serving program keeps the keys and values of all its requests in one pool of pages, each of `page` tokens: blocks
[n_pages][heads][page][64 bytes] and meta words [n_pages][heads][page] in the two-chain format of include/ecco.h.  In every
step it
  take     gives each request the pages that its new tokens need, and learns where each token goes (block table, slots)
  release  gets the pages of requests that are done, or of tokens that were taken back, into the list of free pages again
  append   compresses the new tokens' keys and values into their slots, a chunk of any length per request
  attend   lets the new tokens attend over their request's pages: one token, a few drafted ones, a chunk of a prompt, or
           some of each, each token seeing what is at its position or before it

Each case is a dict of plain values.  The lengths of a case's requests follow from the case alone ("shape" seeds them), all
values from the seed that `prepare` is given; they are distributed as in paper_2505_06901_amd/workloads.py (keys with
per-channel magnitudes, values without).  `own` False: plain torch operations in 32 bits (whole numbers in 64).
"""
import functools
import random

import numpy as np
import torch

import paper_2505_06901_amd as E
from paper_2505_06901_amd import workloads as W

own = False

GROUP = 128


def listed():
    return [
        # eight requests decode a token each: launch and host latency
        {"name": "take_step", "kind": "take", "B": 8, "page": 32, "T": 4096, "new": "one", "short": False, "shape": 1},
        # the prompts of 256 requests are admitted together
        {"name": "take_prompts", "kind": "take", "B": 256, "page": 16, "T": 2048, "new": "chunk", "short": False, "shape": 2},
        # some of 256 requests are done, some give back drafted tokens
        {"name": "release_mixed", "kind": "release", "B": 256, "page": 16, "T": 4096, "shape": 3},
        # a token of each of eight sequences, 32 heads, compressed with every pattern tried
        {"name": "append_step", "kind": "append", "tokens": 8, "H": 32, "page": 32, "selector": "full", "S": 64, "fused": False},
        # a chunk of 2048 tokens, 8 heads, out of the fused projection of queries, keys and values, the online selector
        {"name": "append_chunk", "kind": "append", "tokens": 2048, "H": 8, "page": 16, "selector": "minmax", "S": 16, "fused": True},
        # a long prompt with every pattern tried
        {"name": "append_prompt", "kind": "append", "tokens": 4096, "H": 8, "page": 64, "selector": "full", "S": 64, "fused": True},
        # one short request alone: latency
        {"name": "attend_one", "kind": "attend", "B": 1, "Hq": 32, "Hkv": 8, "page": 16, "T": 300, "new": "one", "most": 1, "half": False, "S": 16, "shape": 7},
        # one decoding step, grouped queries, requests of different lengths
        {"name": "attend_step", "kind": "attend", "B": 8, "Hq": 32, "Hkv": 8, "page": 32, "T": 4096, "new": "one", "most": 1, "half": False, "S": 16, "shape": 8},
        # one decoding step with a cache per query head
        {"name": "attend_step_heads", "kind": "attend", "B": 8, "Hq": 32, "Hkv": 32, "page": 64, "T": 4096, "new": "one", "most": 1, "half": True, "S": 64, "shape": 9},
        # five drafted tokens of each request, to be verified
        {"name": "attend_drafts", "kind": "attend", "B": 8, "Hq": 32, "Hkv": 8, "page": 16, "T": 4096, "new": "drafts", "most": 5, "half": False, "S": 16, "shape": 10},
        # chunks of two prompts beside six requests that decode
        {"name": "attend_mixed", "kind": "attend", "B": 8, "Hq": 32, "Hkv": 8, "page": 32, "T": 4096, "new": "mixed", "most": 512, "half": False, "S": 16, "shape": 11},
        # the second half of a long prompt
        {"name": "attend_prompt", "kind": "attend", "B": 1, "Hq": 32, "Hkv": 8, "page": 64, "T": 8192, "new": "chunk", "most": 4096, "half": True, "S": 64, "shape": 12},
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread evenly over the logarithm."""
    return max(lo, min(hi, int(round(float(lo) * (float(hi) / lo) ** rng.random()))))


def draw(rng):
    kind = rng.choice(["take", "release", "append", "append", "attend", "attend", "attend", "attend"])
    page, shape = rng.choice([16, 32, 64, 128]), rng.randrange(1 << 30)
    if kind == "take":
        return {"kind": kind, "B": _log(rng, 1, 512), "page": page, "T": _log(rng, 64, 4096), "new": rng.choice(["one", "drafts", "mixed", "chunk"]),
                "short": rng.random() < 0.25, "shape": shape}
    if kind == "release":
        return {"kind": kind, "B": _log(rng, 1, 512), "page": page, "T": _log(rng, 64, 4096), "shape": shape}
    if kind == "append":
        H, selector = rng.choice([4, 8, 16, 32]), rng.choice(["full", "minmax"])
        return {"kind": kind, "tokens": _log(rng, 1, 32768 // H), "H": H, "page": page, "selector": selector, "S": rng.choice([16, 64]), "fused": rng.random() < 0.5}
    B, Hkv, grp, new = _log(rng, 1, 32), rng.choice([4, 8, 16, 32]), rng.choice([1, 2, 4, 8]), rng.choice(["one", "drafts", "mixed", "chunk"])
    T = _log(rng, 16, min(32768, 8 * 32 * 4096 // (B * Hkv)))
    # no more products than the largest listed case has
    most = {"one": 1, "drafts": rng.randint(2, 8)}.get(new) or _log(rng, 16, 4096)
    most = max(1, min(most, T, 32 * 4096 * 6144 // (Hkv * grp * T * (B if new == "chunk" else (B + 3) // 4))))
    return {"kind": kind, "B": B, "Hq": Hkv * grp, "Hkv": Hkv, "page": page, "T": T, "new": new, "most": most, "half": rng.random() < 0.5, "S": rng.choice([16, 64]),
            "shape": shape}


# ---- the requests' lengths, from the case alone ---------------------------------------------------------------------
def _lengths(case):
    """(tokens already held, new tokens) of every request."""
    rng, T, B = random.Random(case["shape"]), case["T"], case["B"]
    held, new = [], []
    for b in range(B):
        most = case.get("most") or min(T, 512)
        if case["new"] == "one":
            n = 1
        elif case["new"] == "drafts":
            n = min(case.get("most", 5), T)
        elif case["new"] == "mixed":  # every fourth a chunk, the first among them
            n = max(1, most - rng.randrange(most // 8 + 1)) if b % 4 == 0 else 1
        else:
            n = max(1, most - (rng.randrange(most // 4 + 1) if B > 1 else 0))
        n = min(n, T)
        total = T if B == 1 or (case["kind"] == "attend" and case["Hq"] == case["Hkv"]) else rng.randint(max(n, T // 8), T)
        held.append(max(0, total - n))
        new.append(n)
    return held, new


def _pages(tokens, page):
    return (tokens + page - 1) // page


# ---- what a program keeps: models fitted once, on calibration data, and uploaded ------------------------------------
@functools.lru_cache(maxsize=None)
def _model(which, S):
    k, v = W.kv_cache(1, 32, 64, GROUP, seed=3)
    return E.ecco_model_to_device(E.ecco_fit_patterns(k if which == "key" else v, S, 12, 3), 0)


@functools.lru_cache(maxsize=None)
def _key_channels(heads):
    """The per-channel magnitudes of the calibration keys, [heads][128]."""
    a = 10.0 ** (2.0 * W.uniform01(3, 20, 0, 32 * GROUP) - 1.0)
    return torch.from_numpy(np.ascontiguousarray(a.reshape(32, GROUP)[:heads]).astype(np.float32)).cuda()


def _ints(a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


def _table(gen, lens, page, max_pages, n_pages):
    """A block table of pages in random order, and the pages that nobody holds."""
    order = torch.randperm(n_pages, device="cuda", generator=gen).to(torch.int32)
    n = torch.tensor([_pages(x, page) for x in lens], device="cuda")
    col = torch.arange(max_pages, device="cuda")
    used = col[None, :] < n[:, None]
    at = (torch.cumsum(n, 0) - n)[:, None] + col[None, :]
    table = torch.where(used, order[at.clamp(max=n_pages - 1)], torch.full_like(order[:1], -1))
    return table.contiguous(), order[int(n.sum()):]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    kind, page = case["kind"], case["page"]
    s = {"case": case}
    if kind in ("take", "release"):
        T, B = case["T"], case["B"]
        s["max_pages"] = _pages(T, page) + 1
        if kind == "take":
            held, new = _lengths(case)
            after = [h + n for h, n in zip(held, new)]
        else:
            rng = random.Random(case["shape"])
            held = [rng.randint(0, T) for _ in range(B)]
            after = held
            # a quarter done, half as they are, a quarter a few tokens shorter
            s["keep"] = _ints([rng.choice([0, h, h, max(0, h - rng.randint(1, 8))]) for h in held])
        need = sum(_pages(a, page) - _pages(h, page) for a, h in zip(after, held))
        n_pages = sum(_pages(a, page) for a in after) + 64
        s["table"], free = _table(gen, held, page, s["max_pages"], n_pages)
        s["held"], s["n_pages"] = _ints(held), n_pages
        s["free"] = torch.full((n_pages,), -1, dtype=torch.int32, device="cuda")
        s["free"][:free.numel()] = free
        count = free.numel()
        if kind == "take":
            if case["short"]:
                count = (2 * need) // 3
            s["new"], s["n_tokens"] = _ints(new), sum(new)
            s["q_start"], s["kv_len"] = _ints([0] * (B + 1)), _ints([0] * B)
            s["slots"] = _ints([0] * s["n_tokens"])
        s["count"], s["left"] = _ints([count]), _ints([0])
        return s
    S = case["S"]
    s["mk"], s["mv"] = _model("key", S), _model("value", S)
    if kind == "append":
        n, H = case["tokens"], case["H"]
        n_pages = _pages(n, page) + 8
        width = (4 * H + 2 * H) * GROUP if case["fused"] else H * GROUP
        x = torch.randn(n, width if case["fused"] else 2 * width, device="cuda", generator=gen)
        at = 4 * H * GROUP if case["fused"] else 0
        x[:, at:at + H * GROUP] *= _key_channels(H).reshape(1, -1)
        x = x.to(torch.float16)
        k, v = x[:, at:at + H * GROUP], x[:, at + H * GROUP:at + 2 * H * GROUP]
        if not case["fused"]:
            k, v = k.contiguous(), v.contiguous()
        s["k"], s["v"] = k.unflatten(1, (H, GROUP)), v.unflatten(1, (H, GROUP))
        order = torch.randperm(n_pages, device="cuda", generator=gen)
        first = 5 % page  # the chunk begins inside a page
        t = torch.arange(n, device="cuda") + first
        s["slots"] = (order[t // page] * page + t % page).to(torch.int32)
        for name in ("k", "v"):
            s[name + "b"] = torch.randint(0, 256, (n_pages, H, page, 64), dtype=torch.uint8, device="cuda", generator=gen)
            s[name + "m"] = torch.randint(0, 1 << 22, (n_pages, H, page), dtype=torch.int32, device="cuda", generator=gen)
        return s
    Hq, Hkv = case["Hq"], case["Hkv"]
    held, new = _lengths(case)
    total = [h + n for h, n in zip(held, new)]
    n_pages, max_pages, n_tokens = sum(_pages(t, page) for t in total) + 8, _pages(case["T"], page), sum(new)
    s["table"], _ = _table(gen, total, page, max_pages, n_pages)
    s["q_start"], s["kv_len"] = _ints(np.concatenate([[0], np.cumsum(new)]).tolist()), _ints(total)
    s["max_new"], s["max_kv"], s["total_kv"], s["spans"] = max(new), max(total), sum(total), list(zip(new, total))
    k = torch.randn(n_pages, Hkv, page, GROUP, device="cuda", generator=gen).mul_(_key_channels(Hkv).view(1, Hkv, 1, GROUP)).to(torch.float16)
    s["kb"], s["km"] = E.ecco_encode(s["mk"], k)
    k = torch.randn(n_pages, Hkv, page, GROUP, device="cuda", generator=gen).to(torch.float16)
    s["vb"], s["vm"] = E.ecco_encode(s["mv"], k)
    for name in ("k", "v"):
        s[name + "b"] = s[name + "b"].view(n_pages, Hkv, page, 64)
        s[name + "m"] = s[name + "m"].view(n_pages, Hkv, page)
    s["q"] = torch.randn(n_tokens, Hq, GROUP, device="cuda", generator=gen).to(torch.float16)
    s["out"] = torch.empty((n_tokens, Hq, GROUP), dtype=torch.float16 if case["half"] else torch.float32, device="cuda")
    return s


# ---- the pages, plain -----------------------------------------------------------------------------------------------
def _plain_take(s):
    page, n_tokens, max_pages = s["case"]["page"], s["n_tokens"], s["max_pages"]
    held, new, count = s["held"].long(), s["new"].long(), s["count"].long()
    cum = torch.cumsum(new, 0)
    first, last = (held + page - 1) // page, (held + new + page - 1) // page
    fits = (cum <= n_tokens) & (last <= max_pages)
    need = (last - first) * fits
    taken = torch.cumsum(need, 0)
    served = fits & ((need == 0) | (taken <= count))
    col = torch.arange(max_pages, device="cuda")[None, :]
    fresh = (col >= first[:, None]) & (col < last[:, None]) & served[:, None]
    at = count - 1 - ((taken - need)[:, None] + col - first[:, None])
    s["table"].copy_(torch.where(fresh, s["free"][at.clamp(0, s["n_pages"] - 1)], s["table"]))
    s["left"].copy_(count - (need * served).sum())
    s["kv_len"].copy_((held + new) * served)
    s["q_start"].copy_(torch.cat([torch.zeros_like(cum[:1]), cum]).clamp(max=n_tokens))
    t = torch.arange(n_tokens, device="cuda")
    b = torch.searchsorted(cum, t, right=True)
    there = b < cum.numel()
    b = b.clamp(max=cum.numel() - 1)
    pos = held[b] + t - (cum - new)[b]
    p = s["table"][b, (pos // page).clamp(max=max_pages - 1)].long()
    ok = there & served[b] & (p >= 0) & (p < s["n_pages"])
    s["slots"].copy_(torch.where(ok, p * page + pos % page, torch.full_like(p, -1)))


def _plain_release(s):
    page, n = s["case"]["page"], s["n_pages"]
    held, keep, count = s["held"].long(), s["keep"].long(), s["count"].long()
    keep = torch.minimum(keep.clamp(min=0), held)
    col = torch.arange(s["max_pages"], device="cuda")[None, :]
    given = (col >= ((keep + page - 1) // page)[:, None]) & (col < ((held + page - 1) // page)[:, None]) & (s["table"] >= 0) & (s["table"] < n)
    given, pages = given.flatten(), s["table"].flatten()
    at = count + torch.cumsum(given, 0) - 1
    at = torch.where(given & (at < n), at, torch.full_like(at, n))
    longer = torch.cat([s["free"], s["free"][:1]])
    longer.scatter_(0, at, pages)
    s["free"].copy_(longer[:n])
    s["left"].copy_((count + given.sum()).clamp(max=n))


# ---- the block format, plain ----------------------------------------------------------------------------------------
@functools.lru_cache(maxsize=None)
def _tables(m):
    """(centroids [S, 16] FP32, code lengths, canonical codes [S, 16], and for every 12-bit peek its index and length [S, 4096])."""
    cent, lens = m.centroids.view(np.float16).astype(np.float32), m.code_lens.astype(np.int64)
    codes, index, length = np.zeros_like(lens), np.zeros((len(lens), 4096), np.int64), np.zeros((len(lens), 4096), np.int64)
    for p, row in enumerate(lens):
        code = last = 0
        for k in sorted(range(16), key=lambda k: (row[k], k)):
            code <<= int(row[k]) - last
            last = int(row[k])
            codes[p, k] = code
            index[p, code << (12 - last):(code + 1) << (12 - last)] = k
            length[p, code << (12 - last):(code + 1) << (12 - last)] = last
            code += 1
    return tuple(torch.from_numpy(a).cuda() for a in (cent, lens, codes, index, length))


def _plain_decode(m, blocks, meta):
    """[n, 64] bytes and [n] meta words -> [n, 128] FP32 values."""
    cent, _, _, index, length = _tables(m)
    n, meta = meta.numel(), meta.flatten().long() & 0xFFFFFFFF
    words = blocks.reshape(n, 64).view(torch.int32).long() & 0xFFFFFFFF
    words = torch.cat([words, torch.zeros_like(words[:, :3])], 1)
    p = ((meta >> 16) & 63).clamp(max=cent.shape[0] - 1)
    raw, scale = (meta >> 22) & 1, (meta & 0xFFFF).to(torch.int16).view(torch.float16).float()
    pos = torch.stack([torch.zeros_like(meta), torch.where(raw == 1, 256, meta >> 23)], 1)
    found = torch.empty((64, n, 2), dtype=torch.int64, device="cuda")
    for i in range(64):  # a code's place is known when the one before it has been read
        w = (pos >> 5).clamp(max=17)
        both = (torch.gather(words, 1, w) << 32) | torch.gather(words, 1, w + 1)
        peek = (both >> (52 - (pos & 31))) & 4095
        found[i] = torch.where(raw[:, None] == 1, peek >> 8, index[p[:, None], peek])
        pos = (pos + torch.where(raw[:, None] == 1, 4, length[p[:, None], peek])).clamp(max=544)
    found = found.permute(1, 2, 0).reshape(n, GROUP)
    return (torch.gather(cent[p], 1, found) * scale[:, None]).half().float()


def _lowest(d):
    """Index of the least along the last axis, the lowest on a tie."""
    k = torch.arange(d.shape[-1], device="cuda")
    return torch.where(d == d.amin(-1, keepdim=True), k, d.shape[-1]).amin(-1)


def _plain_encode(m, x, selector):
    """[n, 128] FP16 -> blocks as [n, 16] words and [n] meta words."""
    cent, lens, codes, _, _ = _tables(m)
    S, x = cent.shape[0], x.float()
    scale = x.abs().amax(1)
    ends = (cent[None] * scale[:, None, None]).half().float()
    if selector == "minmax":
        lo, hi = x.amin(1)[:, None] - ends[:, :, 0], x.amax(1)[:, None] - ends[:, :, 15]
        p = _lowest(lo * lo + hi * hi)
    else:
        error = torch.empty((x.shape[0], S), device="cuda")
        for j in range(S):  # a pattern at a time: all of them together would not fit
            d = (x[:, :, None] - ends[:, j, None, :]).abs().amin(-1)
            d = d * d
            while d.shape[1] > 1:
                d = d[:, ::2] + d[:, 1::2]
            error[:, j] = d[:, 0]
        p = _lowest(error)
    idx = _lowest((x[:, :, None] - torch.gather(ends, 1, p[:, None, None].expand(-1, 1, 16))).abs())
    bits, code = torch.gather(lens[p], 1, idx), torch.gather(codes[p], 1, idx)
    end = torch.cumsum(bits, 1)
    raw, at = end[:, -1] > 512, end - bits
    both = code << (64 - bits - (at & 31))
    words, w = torch.zeros((x.shape[0], 50), dtype=torch.int64, device="cuda"), at >> 5
    words.scatter_add_(1, w, (both >> 32) & 0xFFFFFFFF)
    words.scatter_add_(1, w + 1, both & 0xFFFFFFFF)
    shift = 28 - 4 * torch.arange(8, device="cuda")
    words = torch.where(raw[:, None], (idx.view(-1, 16, 8) << shift).sum(-1), words[:, :16])
    meta = scale.half().view(torch.int16).long() | (p << 16) | (raw.long() << 22) | (torch.where(raw, 256, end[:, 63]) << 23)
    return words.to(torch.int32), meta.to(torch.int32)


def _plain_append(s):
    c, slots, done = s["case"], s["slots"].long(), []
    for x, m, blocks, meta in ((s["k"], s["mk"], s["kb"], s["km"]), (s["v"], s["mv"], s["vb"], s["vm"])):
        n_pages, H, page = meta.shape
        groups = x.reshape(-1, GROUP)
        parts = [_plain_encode(m, g, c["selector"]) for g in groups.split(16384)]
        words, mw = torch.cat([a for a, _ in parts]).view(-1, H, 16), torch.cat([a for _, a in parts]).view(-1, H)
        # the token that each slot of the pool takes, if any
        source = torch.full((n_pages * page + 1,), -1, device="cuda")
        source.scatter_(0, torch.where((slots >= 0) & (slots < n_pages * page), slots, n_pages * page), torch.arange(slots.numel(), device="cuda"))
        source = source[:-1].view(n_pages, 1, page).expand(n_pages, H, page)
        head = torch.arange(H, device="cuda")[None, :, None]
        old = blocks.view(torch.int32)
        old.copy_(torch.where(source[..., None] >= 0, words[source.clamp(min=0), head], old))
        meta.copy_(torch.where(source >= 0, mw[source.clamp(min=0), head], meta))
        done += [old, meta]
    return done


# ---- attention, plain -----------------------------------------------------------------------------------------------
def _request(s, b, total):
    """The blocks of request b's tokens in order: [heads, total, 64] and [heads, total], of the keys and of the values."""
    page = s["case"]["page"]
    rows = s["table"][b, :_pages(total, page)].long()
    return [s[n][rows].transpose(0, 1).flatten(1, 2)[:, :total] for n in ("kb", "km", "vb", "vm")]


def _plain_attend(s):
    Hkv, row = s["case"]["Hkv"], 0
    for b, (n, total) in enumerate(s["spans"]):
        kb, km, vb, vm = _request(s, b, total)
        k, v = _plain_decode(s["mk"], kb, km).view(Hkv, total, GROUP), _plain_decode(s["mv"], vb, vm).view(Hkv, total, GROUP)
        q = s["q"][row:row + n].float().unflatten(1, (Hkv, -1)).permute(1, 0, 2, 3)  # [Hkv, n, group, 128]
        grp = q.shape[2]
        score = torch.matmul(q.reshape(Hkv, n * grp, GROUP), k.transpose(1, 2).contiguous()) * GROUP ** -0.5
        seen = torch.arange(total, device="cuda")[None, :] <= (total - n + torch.arange(n, device="cuda"))[:, None]
        score = score.view(Hkv, n, grp, total).masked_fill_(~seen[None, :, None, :], float("-inf"))
        p = torch.exp(score - score.amax(-1, keepdim=True)).view(Hkv, n * grp, total)
        o = torch.matmul(p, v) / p.sum(-1, keepdim=True)
        s["out"][row:row + n] = o.view(Hkv, n, grp, GROUP).permute(1, 0, 2, 3).reshape(n, -1, GROUP).to(s["out"].dtype)
        row += n
    return s["out"]


def run(s):
    c = s["case"]
    if c["kind"] == "take":
        if own:
            E.ecco_kv_pages_take(s["held"], s["new"], s["table"], s["free"], s["count"], c["page"], s["n_tokens"], s["left"], s["q_start"], s["kv_len"], s["slots"])
        else:
            _plain_take(s)
        return {k: s[k] for k in ("table", "left", "q_start", "kv_len", "slots")}
    if c["kind"] == "release":
        if own:
            E.ecco_kv_pages_release(s["held"], s["keep"], s["table"], s["free"], s["count"], c["page"], s["left"])
        else:
            _plain_release(s)
        return {k: s[k] for k in ("free", "left")}
    if c["kind"] == "append":
        if own:
            call = E.ecco_kv_append_paged if c["selector"] == "full" else E.ecco_kv_append_paged_minmax
            call(s["mk"], s["mv"], s["k"], s["v"], s["kb"], s["km"], s["vb"], s["vm"], s["slots"])
            return [s["kb"].view(torch.int32), s["km"], s["vb"].view(torch.int32), s["vm"]]
        return _plain_append(s)
    if own:
        if "workspace" not in s:  # kept by a program as long as its sizes stay
            s["workspace"] = torch.empty((E.ecco_kv_attend_paged_workspace(s["q"].shape[0], c["B"], c["Hq"], c["Hkv"], s["max_new"], s["max_kv"], s["total_kv"]),),
                                         dtype=torch.uint8, device="cuda")
        return E.ecco_kv_attend_paged(s["mk"], s["mv"], s["q"], s["kb"], s["km"], s["vb"], s["vm"], s["table"], s["q_start"], s["kv_len"], s["max_new"], s["max_kv"],
                                      s["total_kv"], s["workspace"], s["out"])
    return _plain_attend(s)


def work(case):
    kind, page = case["kind"], case["page"]
    if kind == "take":
        held, new = _lengths(case)
        pages = sum(_pages(h + n, page) - _pages(h, page) for h, n in zip(held, new))
        return {"bytes": 4 * (4 * case["B"] + 2 * pages + sum(new) + 3), "flops": 0}
    if kind == "release":
        rng = random.Random(case["shape"])
        held = [rng.randint(0, case["T"]) for _ in range(case["B"])]
        keep = [rng.choice([0, h, h, max(0, h - rng.randint(1, 8))]) for h in held]
        return {"bytes": 4 * (2 * case["B"] + 2 * sum(_pages(h, page) - _pages(k, page) for h, k in zip(held, keep)) + 2), "flops": 0}
    if kind == "append":
        n, S = 2 * case["tokens"] * case["H"], case["S"]
        # the search over all patterns: a subtraction and a comparison per value, centroid and pattern, squared and summed
        per = GROUP * (16 * 2 + 2)
        return {"bytes": n * (2 * GROUP + 64 + 4) + 4 * case["tokens"], "flops": n * per * (S if case["selector"] == "full" else 1)}
    held, new = _lengths(case)
    seen = sum(n * h + n * (n + 1) // 2 for h, n in zip(held, new))
    tokens, rows = sum(held) + sum(new), sum(new) * case["Hq"]
    return {"bytes": 2 * tokens * case["Hkv"] * 68 + rows * GROUP * (2 + (2 if case["half"] else 4)) + 4 * sum(_pages(h + n, page) for h, n in zip(held, new)),
            "flops": 4 * GROUP * case["Hq"] * seen}


# ---- from the definitions, in 64 bits --------------------------------------------------------------------------------
def _exact_take(s):
    page, held, new = s["case"]["page"], s["held"].tolist(), s["new"].tolist()
    table, free, count = s["table"].tolist(), s["free"].tolist(), int(s["count"][0])
    starts, lens, slots, rows, asked, gone = [0], [], [], 0, 0, 0
    for b, (h, n) in enumerate(zip(held, new)):
        have, want = -(-h // page), -(-(h + n) // page)
        fits = rows + n <= s["n_tokens"] and want <= s["max_pages"]
        asked += want - have if fits else 0
        good = fits and (want == have or asked <= count)
        if good:
            for i in range(have, want):
                gone += 1
                table[b][i] = free[count - gone]
        for t in range(h, h + n):
            at = table[b][t // page] if good else -1
            slots.append(at * page + t % page if 0 <= at < s["n_pages"] else -1)
        rows += n
        starts.append(min(rows, s["n_tokens"]))
        lens.append(h + n if good else 0)
    slots = (slots + [-1] * s["n_tokens"])[:s["n_tokens"]]
    return {"table": _ints(table), "left": _ints([count - gone]), "q_start": _ints(starts), "kv_len": _ints(lens), "slots": _ints(slots)}


def _exact_release(s):
    page, free, count = s["case"]["page"], s["free"].tolist(), int(s["count"][0])
    for row, h, k in zip(s["table"].tolist(), s["held"].tolist(), s["keep"].tolist()):
        for i in range(-(-min(max(k, 0), h) // page), -(-h // page)):
            if 0 <= row[i] < s["n_pages"] and count < s["n_pages"]:
                free[count] = row[i]
                count += 1
    return {"free": _ints(free), "left": _ints([count])}


def _canonical(lens):
    """Symbols by (length, symbol), and for each the code, left-aligned in 12 bits."""
    order, at = [], []
    for row in lens.tolist():
        o = sorted(range(16), key=lambda k: (row[k], k))
        ends = np.cumsum([1 << (12 - row[k]) for k in o])
        order.append(o)
        at.append([0] + ends[:-1].tolist())
    return torch.tensor(order, device="cuda"), torch.tensor(at, device="cuda")


def _exact_decode(m, blocks, meta):
    """One stream of 128 codes, bit by bit out of the 512."""
    order, at = _canonical(m.code_lens)
    lens = torch.from_numpy(m.code_lens.astype(np.int64)).cuda()
    cent = torch.from_numpy(m.centroids.view(np.float16).astype(np.float64)).cuda()
    meta = meta.reshape(-1).cpu().numpy().view(np.uint32).astype(np.int64)
    scale = torch.from_numpy((meta & 0xFFFF).astype(np.uint16).view(np.float16).astype(np.float64)).cuda()
    p, raw = torch.from_numpy(np.minimum((meta >> 16) & 63, len(m.code_lens) - 1)).cuda(), torch.from_numpy((meta >> 22) & 1).cuda().bool()
    n = len(meta)
    swapped = blocks.reshape(n, 16, 4).flip(2).reshape(n, 64)  # the most significant byte of each word first
    bit = torch.arange(7, -1, -1, device="cuda", dtype=torch.uint8)
    bits = ((swapped[:, :, None] >> bit) & 1).view(n, 512)
    bits = torch.cat([bits, torch.zeros_like(bits[:, :16])], 1)
    pos, weight, out = torch.zeros(n, dtype=torch.int64, device="cuda"), 1 << torch.arange(11, -1, -1, device="cuda"), []
    for _ in range(GROUP):
        peek = (torch.gather(bits, 1, (pos[:, None] + torch.arange(12, device="cuda")).clamp(max=527)).long() * weight).sum(1)
        rank = (at[p] <= peek[:, None]).sum(1) - 1
        k = torch.where(raw, peek >> 8, order[p, rank])
        out.append(k)
        pos = pos + torch.where(raw, 4, lens[p, k])
    value = torch.gather(cent[p], 1, torch.stack(out, 1)) * scale[:, None]  # exact in 64 bits
    return value.to(torch.float16).double()


def _to32(x):
    return x.to(torch.float32).double()


def _exact_encode(m, x, selector):
    """The definition's FP32 operations as 64-bit ones, each rounded."""
    order, at = _canonical(m.code_lens)
    lens = torch.from_numpy(m.code_lens.astype(np.int64)).cuda()
    cent = torch.from_numpy(m.centroids.view(np.float16).astype(np.float64)).cuda()
    x = x.double()
    scale = x.abs().max(1).values
    least, p = torch.full_like(scale, float("inf")), torch.zeros_like(scale, dtype=torch.int64)
    for j in range(cent.shape[0]):
        r = (cent[j] * scale[:, None]).to(torch.float16).double()
        if selector == "minmax":
            lo, hi = _to32(x.min(1).values - r[:, 0]), _to32(x.max(1).values - r[:, 15])
            e = _to32(_to32(lo * lo) + _to32(hi * hi))
        else:
            d = torch.full_like(x, float("inf"))
            for k in range(16):
                d = torch.minimum(d, _to32(x - r[:, k:k + 1]).abs())
            e = _to32(d * d)
            for step in (1, 2, 4, 8, 16, 32, 64):
                e = _to32(e + e[:, torch.arange(GROUP, device="cuda") ^ step])
            e = e[:, 0]
        better = e < least
        least, p = torch.where(better, e, least), torch.where(better, j, p)
    r = (cent[p] * scale[:, None]).to(torch.float16).double()
    best, idx = torch.full_like(x, float("inf")), torch.zeros_like(x, dtype=torch.int64)
    for k in range(16):
        d = _to32(x - r[:, k:k + 1]).abs()
        idx, best = torch.where(d < best, k, idx), torch.minimum(d, best)
    code = torch.zeros_like(lens).scatter_(1, order, at)  # left-aligned in 12 bits
    n = torch.gather(lens[p], 1, idx)
    digit = torch.arange(12, device="cuda")
    there = (digit < n[:, :, None]).flatten(1)
    value = ((torch.gather(code[p], 1, idx)[:, :, None] >> (11 - digit)) & 1).flatten(1)
    place = torch.cumsum(there, 1) - 1
    total, middle = n.sum(1), n[:, :64].sum(1)
    bits = torch.zeros((x.shape[0], 128 * 12 + 1), dtype=torch.int64, device="cuda")
    bits.scatter_(1, torch.where(there, place, 128 * 12), value)
    plain = ((idx[:, :, None] >> torch.arange(3, -1, -1, device="cuda")) & 1).flatten(1)
    raw = total > 512
    bits = torch.where(raw[:, None], plain, bits[:, :512]).view(-1, 16, 32)
    words = (bits << torch.arange(31, -1, -1, device="cuda")).sum(-1)
    meta = scale.half().view(torch.int16).long() + p * 65536 + raw.long() * (1 << 22) + torch.where(raw, 256, middle) * (1 << 23)
    return words.to(torch.int32), meta.to(torch.int32)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "take":
        return _exact_take(s)
    if case["kind"] == "release":
        return _exact_release(s)
    if case["kind"] == "append":
        out = []
        for x, m, blocks, meta in ((s["k"], s["mk"], s["kb"], s["km"]), (s["v"], s["mv"], s["vb"], s["vm"])):
            H, page = meta.shape[1:]
            parts = [_exact_encode(m, g, case["selector"]) for g in x.reshape(-1, GROUP).split(4096)]
            slots = s["slots"].long()
            at = ((slots // page * H)[:, None] + torch.arange(H, device="cuda")) * page + (slots % page)[:, None]
            blocks, meta = blocks.view(torch.int32).clone(), meta.clone()
            blocks.view(-1, 16)[at.flatten()] = torch.cat([a for a, _ in parts])
            meta.view(-1)[at.flatten()] = torch.cat([a for _, a in parts])
            out += [blocks, meta]
        return out
    Hkv, grp, row = case["Hkv"], case["Hq"] // case["Hkv"], 0
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    for b, (n, total) in enumerate(s["spans"]):
        kb, km, vb, vm = _request(s, b, total)
        last = total - n + torch.arange(n, device="cuda").repeat_interleave(grp)
        hidden = torch.arange(total, device="cuda")[None, :] > last[:, None]
        for h in range(Hkv):
            q = s["q"][row:row + n, h * grp:(h + 1) * grp].double().reshape(n * grp, GROUP)
            k, v = _exact_decode(s["mk"], kb[h], km[h]), _exact_decode(s["mv"], vb[h], vm[h])
            p = torch.softmax((q @ k.T / 128.0 ** 0.5).masked_fill(hidden, float("-inf")), -1)
            out[row:row + n, h * grp:(h + 1) * grp] = (p @ v).view(n, grp, GROUP)
        row += n
    return out
