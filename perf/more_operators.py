"""The operators of a serving loop whose requests share and outgrow the paged 4-bit cache: pages forked, written apart, released and
compacted; attention of a batch that shares a long prefix; summaries of pages, the choice of pages for a query by them, and attention over the chosen ones.

`own` chooses who computes: the package's kernels, or the plain forms below, elementary torch operations in 32 bits (whole numbers in
64).  A batch is described the way a serving loop holds it: a page table [sequences, pages], the length of every sequence with its new
tokens (`kv_len`), and where the new tokens of each start in the rows of the call (`q_start`).
"""
from __future__ import annotations

import math
import random

import torch

own = False
DEVICE = "cuda:0"
GROUP = 32                                                               # elements that share a scale in the cache

LLAMA31_8B = {"h_q": 32, "h_kv": 8, "d": 128}
GEMMA2_2B = {"h_q": 8, "h_kv": 4, "d": 256}
HEADS = [LLAMA31_8B, LLAMA31_8B, GEMMA2_2B, {"h_q": 14, "h_kv": 2, "d": 64}, {"h_q": 16, "h_kv": 16, "d": 64}, {"h_q": 12, "h_kv": 1, "d": 128}]


def listed():
    return [
        # one request is continued in four ways: their common pages are shared, each writes its next token to a copy of the last page
        {"name": "fork_1_into_4", "op": "fork", "parents": 1, "children": 4, "longest": 1275, "shortest": 1275, "new": 1, "mix": 0, "page": 16, "spare": 400, **LLAMA31_8B},
        # a batch of users of a few system prompts, large pages, a pool of many
        {"name": "fork_5_into_256", "op": "fork", "parents": 5, "children": 256, "longest": 4001, "shortest": 700, "new": 30, "mix": 4, "page": 64, "spare": 3000, **LLAMA31_8B},
        # half of the requests are done: their pages are given back and the others moved together, a small pool and a large one
        {"name": "compact_12", "op": "compact", "B": 12, "longest": 600, "shortest": 100, "mix": 1, "page": 16, "spare": 50, **GEMMA2_2B},
        {"name": "compact_96", "op": "compact", "B": 96, "longest": 4096, "shortest": 900, "mix": 2, "page": 64, "spare": 500, **LLAMA31_8B},
        # summaries follow a generated token of a batch, and the prompts of one
        {"name": "summaries_64_tokens", "op": "summaries", "B": 64, "longest": 700, "shortest": 300, "new": 1, "mix": 3, "page": 64, **LLAMA31_8B},
        {"name": "summaries_6_prompts", "op": "summaries", "B": 6, "longest": 8192, "shortest": 2000, "new": 0, "mix": 6, "page": 32, **LLAMA31_8B},
        # four samples of one prompt, at the length of the 1024 + 256 token protocol
        {"name": "shared_4_of_1024", "op": "shared", "groups": 1, "B": 4, "prefix": 1024, "longest": 256, "shortest": 256, "new": 1, "mix": 0, "page": 16, "softcap": 0.0, **LLAMA31_8B},
        # a serving batch over one long document
        {"name": "shared_64_of_32768", "op": "shared", "groups": 1, "B": 64, "prefix": 32768, "longest": 1500, "shortest": 20, "new": 1, "mix": 5, "page": 64, "softcap": 0.0, **LLAMA31_8B},
        # three system prompts, wide heads, a soft cap; a few drafted tokens of every request are verified
        {"name": "shared_3_of_8192_drafts", "op": "shared", "groups": 3, "B": 48, "prefix": 8192, "longest": 2000, "shortest": 100, "new": 4, "mix": 7, "page": 32, "softcap": 50.0, **GEMMA2_2B},
        # one user's generated token at the end of a long document: 64 of its 2048 pages
        {"name": "sparse_1_at_131071", "op": "sparse", "B": 1, "longest": 131071, "shortest": 131071, "new": 1, "mix": 0, "page": 64, "budget": 64, "softcap": 0.0, **LLAMA31_8B},
        # a serving batch of ragged lengths, an eighth of the longest one's pages
        {"name": "sparse_32_ragged", "op": "sparse", "B": 32, "longest": 32768, "shortest": 1000, "new": 1, "mix": 8, "page": 32, "budget": 128, "softcap": 0.0, **LLAMA31_8B},
        # wide heads, a soft cap, small pages
        {"name": "sparse_8_of_16000", "op": "sparse", "B": 8, "longest": 16000, "shortest": 16000, "new": 2, "mix": 0, "page": 16, "budget": 100, "softcap": 50.0, **GEMMA2_2B},
    ]


def _log_int(rng, lo, hi, step=1):
    return max(step, round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step) * step)


def draw(rng):
    op = rng.choice(["fork", "compact", "summaries", "shared", "shared", "shared", "sparse", "sparse", "sparse"])
    heads, page, mix = rng.choice(HEADS), rng.choice([16, 32, 64, 128]), rng.randrange(1 << 20)
    case, wide = {"op": op, "mix": mix, "page": page, **heads}, heads["h_kv"] * heads["d"]
    if op == "fork":
        longest = _log_int(rng, 1, 4000)
        children = _log_int(rng, 1, 256)
        new = _log_int(rng, 1, min(200, max(2, 30 * 256 * 1024 // (children * wide))))
        return {**case, "parents": rng.randint(1, min(children, 5)), "children": children, "longest": longest, "shortest": max(1, longest // 4), "new": new, "spare": children * (new // page + 2) + rng.randint(0, 2000)}
    if op == "compact":
        longest = _log_int(rng, 5, 4096)
        return {**case, "B": _log_int(rng, 2, max(2, min(200, 96 * 4096 * 1024 // (2 * longest * wide)))), "longest": longest, "shortest": max(1, longest // 5), "spare": rng.randint(0, 500)}
    if op == "summaries":
        longest = _log_int(rng, 1, 8192)
        return {**case, "B": _log_int(rng, 1, max(1, min(128, 6 * 4096 * 1024 // (longest * wide)))), "longest": longest, "shortest": max(1, longest // 4), "new": rng.choice([0, 1, 1, 7])}
    case["softcap"] = rng.choice([0.0, 0.0, 0.0, 50.0])
    if op == "shared":
        new = rng.choice([1, 1, 1, rng.randint(2, 8)])
        prefix = _log_int(rng, page, 32768, page)
        most = max(2, min(128, 64 * 32768 * 32 // (prefix * heads["h_q"] * new)))
        B, longest = _log_int(rng, 2, most), _log_int(rng, new, 1500)
        return {**case, "groups": rng.randint(1, min(4, max(1, B // 2))), "B": B, "prefix": prefix, "longest": longest, "shortest": max(new, longest // rng.choice([1, 4, 16])), "new": new}
    longest = _log_int(rng, 10, 100000)
    budget = rng.choice([_log_int(rng, 4, 4096 // page * 2), 32])
    most = max(1, min(64, 32 * 32768 * 1024 // (longest * wide), 32 * 4096 * 1024 // (min(longest, budget * page) * wide)))
    return {**case, "B": _log_int(rng, 1, most), "longest": longest, "shortest": max(1, longest // rng.choice([1, 4, 16])), "new": rng.choice([1, 1, 1, 3]), "budget": budget}


# ---------------------------------------------------------------------------- what a case holds
def _lengths(case):
    """Length of every sequence: the first is the longest, the others are spread over the logarithm."""
    rng = random.Random(case["mix"])
    n = case["parents"] if case["op"] == "fork" else case["B"]
    return [case["longest"]] + [_log_int(rng, case["shortest"], case["longest"]) for _ in range(n - 1)]


def _batch(case):
    """(length with the new tokens, new tokens) of every sequence of a call."""
    lens = _lengths(case)
    if case["op"] == "shared":
        return [case["prefix"] + n for n in lens], [min(case["new"], n) for n in lens]
    return lens, [n if case["new"] == 0 else min(case["new"], n) for n in lens]


def _group_of(case):
    """The group of every sequence of a shared call: as many sequences each as there are, to one."""
    return [b * case["groups"] // case["B"] for b in range(case["B"])]


def _starts(counts):
    return [sum(counts[:i]) for i in range(len(counts) + 1)]


def _generator(seed):
    return torch.Generator(device=DEVICE).manual_seed(seed)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEVICE)


def _table(rows, width):
    return _ints([list(r) + [-1] * (width - len(r)) for r in rows])


def prepare(case, seed):
    g, rng = _generator(seed), random.Random(seed)
    s = {"case": case}
    {"fork": _prepare_fork, "compact": _prepare_compact, "summaries": _prepare_call, "shared": _prepare_call, "sparse": _prepare_call}[case["op"]](s, case, g, rng)
    return s


def _fill(s, case, g, n_pages):
    """A pool that is full: the package's cache, or the integers and scales that it stands for."""
    page, h_kv, d = case["page"], case["h_kv"], case["d"]
    slots = n_pages * page
    # keys of a trained model: some channels of a head are several times larger than the others
    channel = torch.exp(0.5 * torch.randn(h_kv * d, generator=g, device=DEVICE)).half()
    k = torch.randn(slots, h_kv * d, generator=g, device=DEVICE, dtype=torch.float16) * channel
    v = torch.randn(slots, h_kv * d, generator=g, device=DEVICE, dtype=torch.float16)
    if case["op"] in ("sparse", "summaries"):                            # a page holds text of one subject: its keys have something in common
        k = (k.view(n_pages, page, -1) + 1.5 * channel * torch.randn(n_pages, 1, h_kv * d, generator=g, device=DEVICE, dtype=torch.float16)).view(slots, -1)
    s["n_pages"] = n_pages
    if own:
        s["cache"] = _package().PagedKV(n_pages, page, h_kv, d, device=DEVICE)
        s["cache"].append(k, v, torch.arange(n_pages, dtype=torch.int32, device=DEVICE)[None, :], _ints([slots]), _ints([0, slots]))
    else:
        s["k_codes"], s["k_scales"] = _to_4_bits(k.view(slots, h_kv, d))
        s["v_codes"], s["v_scales"] = _to_4_bits(v.view(slots, h_kv, d))


def _prepare_fork(s, case, g, rng):
    lens, page, n = _lengths(case), case["page"], case["children"]
    need = [-(-x // page) for x in lens]
    n_pages = sum(need) + case["spare"]
    order = rng.sample(range(n_pages), sum(need))                        # pages in the order in which a busy pool would hand them out
    width = max(-(-(x + case["new"]) // page) for x in lens)
    s["table"] = _table([order[a:b] for a, b in zip(_starts(need), _starts(need)[1:])], width)
    refs = torch.zeros(n_pages, dtype=torch.int32, device=DEVICE)
    refs[order] = 1
    s["refs"] = refs
    parents = [i * case["parents"] // n for i in range(n)]
    s["parents"], s["lengths"] = _ints(parents), _ints([lens[p] for p in parents])
    s["kv_len"] = s["lengths"] + case["new"]
    s["q_start"], s["T"] = _ints([i * case["new"] for i in range(n + 1)]), n * case["new"]
    # what is looked at afterwards: the tokens in front of the new ones in their page
    tail = [(lens[p] - 1) % page + 1 for p in parents]
    s["tail_start"], s["tail"] = _ints(_starts(tail)), sum(tail)
    _fill(s, case, g, n_pages)


def _prepare_compact(s, case, g, rng):
    lens, page = _lengths(case), case["page"]
    need = [-(-x // page) for x in lens]
    n_pages = sum(need) + case["spare"]
    order = rng.sample(range(n_pages), sum(need))
    s["table"] = _table([order[a:b] for a, b in zip(_starts(need), _starts(need)[1:])], max(need))
    s["refs"] = torch.zeros(n_pages, dtype=torch.int32, device=DEVICE)
    s["refs"][order] = 1
    done = sorted(random.Random(case["mix"] + 1).sample(range(case["B"]), case["B"] // 2))
    left = [0 if b in done else n for b, n in enumerate(lens)]
    s["done"], s["left"], s["left_start"], s["T"] = _ints(done), _ints(left), _ints(_starts(left)), sum(left)
    _fill(s, case, g, n_pages)


def _prepare_call(s, case, g, rng):
    lens, new = _batch(case)
    page, B = case["page"], case["B"]
    width = max(-(-n // page) for n in lens)
    if case["op"] == "shared":
        whole = case["prefix"] // page                                   # pages of a prefix: its group's
        group = _group_of(case)
        own_pages = [-(-n // page) - whole for n in lens]
        n_pages = case["groups"] * whole + sum(own_pages) + 3
        order = rng.sample(range(n_pages), n_pages)
        at = [x + case["groups"] * whole for x in _starts(own_pages)]
        rows = [order[group[b] * whole : (group[b] + 1) * whole] + order[at[b] : at[b + 1]] for b in range(B)]
        s["group_start"] = _ints([group.index(i) for i in range(case["groups"])] + [B])
        s["prefix_len"] = _ints([case["prefix"]] * case["groups"])
    else:
        need = [-(-n // page) for n in lens]
        n_pages = sum(need) + 3
        order = rng.sample(range(n_pages), n_pages)
        rows = [order[a:b] for a, b in zip(_starts(need), _starts(need)[1:])]
    # entries behind a sequence's last page hold nothing
    s["table"], s["kv_len"], s["q_start"], s["max_q"], s["T"] = _table(rows, width), _ints(lens), _ints(_starts(new)), max(new), sum(new)
    s["q"] = torch.randn(s["T"], case["h_q"] * case["d"], generator=g, device=DEVICE, dtype=torch.float16)
    _fill(s, case, g, n_pages)
    if case["op"] == "shared":
        return
    h_kv, d = case["h_kv"], case["d"]
    if own:
        s["bounds"] = s["cache"].key_bounds()
    else:
        s["bounds"] = torch.zeros(n_pages, h_kv, 2, d, dtype=torch.int8, device=DEVICE), torch.zeros(n_pages, h_kv, device=DEVICE)
    if case["op"] == "sparse":                                           # (kept up to date by the steps before)
        start = _ints(_starts(lens))
        if own:
            s["cache"].summarise(s["bounds"], s["table"], s["kv_len"], start, sum(lens))
        else:
            _summarise(s, case, s["bounds"], lens)


# ---------------------------------------------------------------------------- one pass
def _package():
    import paper_2505_00232_b200
    return paper_2505_00232_b200


def run(s):
    case = s["case"]
    return {"fork": _run_fork, "compact": _run_compact, "summaries": _run_summaries, "shared": _run_shared, "sparse": _run_sparse}[case["op"]](s, case)


def _run_fork(s, case):
    """The children's page table, who holds which page, how many pages were missing, and what the cache holds in front of the new tokens."""
    refs = s["refs"].clone()
    if own:
        cache = s["cache"]
        table = cache.fork(refs, s["table"], s["parents"], s["lengths"])
        missing = cache.reserve(refs, table, s["kv_len"], s["q_start"], s["T"])
        k, v = cache.read(table, s["lengths"], s["tail_start"], s["tail"])
        return table, refs, missing, k, v
    page, n, W = case["page"], case["children"], s["table"].shape[1]
    column = torch.arange(W, device=DEVICE)
    table = torch.where(column < ((s["lengths"] + page - 1) // page)[:, None], s["table"][s["parents"].long()], -1)
    held = table >= 0
    refs.index_add_(0, table.clamp(min=0).flatten().long(), held.flatten().to(torch.int32))
    # pages that new tokens come to: those without a place, and those that others hold too, get the lowest free ones, in order
    first = s["lengths"] // page
    written = (column >= first[:, None]) & (column <= ((s["kv_len"] - 1) // page)[:, None])
    shared = written & held & (refs[table.clamp(min=0).long()] > 1)
    fresh = written & ~held | shared
    free = torch.argsort((refs > 0).to(torch.int8), stable=True)         # (the free ones first)
    rank = torch.cumsum(fresh.flatten().to(torch.int64), 0).view(n, W)
    missing = (rank[-1, -1] - (refs == 0).sum()).clamp(min=0)
    fresh &= missing == 0
    shared &= missing == 0
    page_of = free[(rank - 1).clamp(0, free.numel() - 1)].to(torch.int32)
    at = first.long().clamp(max=W - 1)[:, None]                          # the page that holds tokens already, of every child: copied whole
    copied = (shared.gather(1, at) & (s["lengths"] % page > 0)[:, None])[:, 0]
    source, target = table.gather(1, at)[:, 0].long(), page_of.gather(1, at)[:, 0].long()
    source = torch.where(copied, source, target)
    for x in ("k_codes", "k_scales", "v_codes", "v_scales"):
        pages = s[x].view(s["n_pages"], page, *s[x].shape[1:])
        pages[target] = torch.where(copied[(...,) + (None,) * (pages.dim() - 1)], pages[source], pages[target])
    refs.index_add_(0, table.clamp(min=0).flatten().long(), -shared.flatten().to(torch.int32))
    refs.index_add_(0, page_of.flatten().long(), fresh.flatten().to(torch.int32))
    table = torch.where(fresh, page_of, table)
    k, v = _tokens(s, case, table, s["lengths"], s["tail_start"], s["tail"])
    return table, refs, missing.to(torch.int32)[None], k, v


def _run_compact(s, case):
    """The page table and who holds which page, where each page went, and what the cache holds of the requests that are left."""
    refs, table = s["refs"].clone(), s["table"].clone()
    if own:
        cache = s["cache"]
        cache.release(refs, table, s["done"])
        moved = cache.compact(refs, table)
        k, v = cache.read(table, s["left"], s["left_start"], s["T"])
        return table, refs, moved, k, v
    page, n = case["page"], s["n_pages"]
    gone = table[s["done"].long()]
    refs.index_add_(0, gone.clamp(min=0).flatten().long(), -(gone >= 0).flatten().to(torch.int32))
    table[s["done"].long()] = -1
    live = refs > 0
    number = torch.arange(n, device=DEVICE)
    n_live = live.sum()
    mover, place = live & (number >= n_live), ~live & (number < n_live)  # as many of the one as of the other
    order = torch.argsort((~place).to(torch.int8), stable=True)          # the free places in front, in order
    target = order[(torch.cumsum(mover.to(torch.int64), 0) - 1).clamp(min=0)]
    moved = torch.where(live, torch.where(mover, target, number), -1)
    scatter = torch.where(live, moved, n)                                # (the dead ones to a place of their own)
    for x in ("k_codes", "k_scales", "v_codes", "v_scales"):             # whole tokens' slots; the old pool is another call's
        pages = s[x].view(n, page, *s[x].shape[1:])
        to = torch.empty((n + 1, *pages.shape[1:]), dtype=pages.dtype, device=DEVICE)
        to.index_copy_(0, scatter, pages)
        s["new_" + x] = to[:n].flatten(0, 1)
    new_refs = torch.zeros(n + 1, dtype=torch.int32, device=DEVICE).index_copy_(0, scatter, refs)[:n]
    new_refs = torch.where(number < n_live, new_refs, 0)
    table = torch.where(table >= 0, moved[table.clamp(min=0).long()].to(torch.int32), -1)
    k, v = _tokens(s, case, table, s["left"], s["left_start"], s["T"], "new_")
    return table, new_refs, moved.to(torch.int32), k, v


def _run_summaries(s, case):
    """The bounds of every page's keys, as the values that they stand for."""
    if own:
        s["cache"].summarise(s["bounds"], s["table"], s["kv_len"], s["q_start"], s["T"])
    else:
        _summarise(s, case, s["bounds"], _batch(case)[1])
    bounds, scales = s["bounds"]
    return bounds.float() * scales[:, :, None, None]


def _summarise(s, case, out, new):
    """Of every page that holds one of the last new[b] tokens of a sequence: the largest and the smallest key element per channel, in 8 bits of the head's largest magnitude, outwards."""
    page, h_kv, d, W = case["page"], case["h_kv"], case["d"], s["table"].shape[1]
    column = torch.arange(W, device=DEVICE)
    first, last = (s["kv_len"] - _ints(new)).clamp(min=0) // page, (s["kv_len"] - 1) // page
    column0 = torch.arange(max((n - 1) // page + 2 for n in new), device=DEVICE)
    at = first[:, None] + column0                                        # [B, touched]
    touched = (at <= last[:, None]).flatten()
    b = torch.arange(len(new), device=DEVICE)[:, None]
    pages = s["table"][b, at.clamp(max=W - 1).long()].flatten().long()
    tokens = (s["kv_len"][:, None] - at * page).clamp(max=page).flatten()   # of the page
    bounds, scales = out
    for some in torch.split(torch.arange(pages.numel(), device=DEVICE), max(1, 2 ** 27 // (page * h_kv * d))):
        p = pages[some].clamp(min=0)
        slot = p[:, None] * page + torch.arange(page, device=DEVICE)
        k = _from_4_bits(s["k_codes"][slot], s["k_scales"][slot]).half().float()                # [n, page, h_kv, d]
        here = (torch.arange(page, device=DEVICE) < tokens[some][:, None])[:, :, None, None]
        hi = torch.where(here, k, -math.inf).amax(1)
        lo = torch.where(here, k, math.inf).amin(1)
        top = torch.maximum(hi, -lo).amax(-1)
        scale = top / torch.full_like(top, 127.0)
        r = torch.where(top > 0, torch.full_like(top, 127.0) / top, 0.0)[..., None]
        code = torch.stack([torch.ceil(hi * r).clamp(max=127), torch.floor(lo * r).clamp(min=-127)], 2).to(torch.int8)
        # (what no new token touches stays)
        p = torch.where(touched[some], p, p.new_tensor(s["n_pages"]))
        bounds.copy_(torch.cat([bounds, bounds[:1]]).index_copy_(0, p, code)[:-1])
        scales.copy_(torch.cat([scales, scales[:1]]).index_copy_(0, p, scale)[:-1])


def _run_shared(s, case):
    if own:
        return s["cache"].attention_shared(s["q"], s["table"], s["kv_len"], s["q_start"], s["max_q"], s["group_start"], s["prefix_len"], softcap=case["softcap"])
    B, page, h_kv, d, T, n_q = case["B"], case["page"], case["h_kv"], case["d"], s["T"], s["max_q"]
    G, P = case["h_q"] // h_kv, case["prefix"]
    lens, _ = _batch(case)
    position, row, sequence = _positions(s)
    q = torch.zeros(B, n_q, h_kv, G, d, device=DEVICE)
    q[sequence, row] = s["q"].view(T, h_kv, G, d).float()
    at = torch.full((B, n_q), -1, device=DEVICE)
    at[sequence, row] = position
    group, out = _group_of(case), torch.empty(B, n_q, h_kv, G, d, device=DEVICE)
    cap = (lambda x: case["softcap"] * torch.tanh(x / case["softcap"])) if case["softcap"] else (lambda x: x)
    for i in range(case["groups"]):
        b0, b1 = group.index(i), B - group[::-1].index(i)
        n, L = b1 - b0, max(lens[b0:b1]) - P
        rows = q[b0:b1].permute(2, 0, 1, 3, 4).reshape(h_kv, n * n_q * G, d)
        key = torch.arange(P, device=DEVICE)
        slot = s["table"][b0].long()[key // page] * page + key % page
        # the prefix, once for all rows of the group
        score = cap(rows @ _from_4_bits(s["k_codes"][slot], s["k_scales"][slot]).permute(1, 2, 0) / math.sqrt(d))
        top = score.amax(-1, keepdim=True)
        score = torch.exp(score - top)
        total, y = score.sum(-1, keepdim=True), score @ _from_4_bits(s["v_codes"][slot], s["v_scales"][slot]).permute(1, 0, 2)
        # each sequence's own tokens
        key = P + torch.arange(L, device=DEVICE)
        slot = s["table"][b0:b1].clamp(min=0).long()[:, key // page] * page + key % page        # [n, L]
        mine = q[b0:b1].permute(0, 2, 1, 3, 4).reshape(n, h_kv, n_q * G, d)
        x = cap(mine @ _from_4_bits(s["k_codes"][slot], s["k_scales"][slot]).permute(0, 2, 3, 1) / math.sqrt(d))
        seen = key[None, None, :] <= at[b0:b1, :, None]
        x = x.view(n, h_kv, n_q, G, L).masked_fill(~seen[:, None, :, None, :], -math.inf).view(n, h_kv, n_q * G, L)
        split = lambda t: t.view(h_kv, n, n_q * G, -1).transpose(0, 1)
        top, total, y = split(top), split(total), split(y)
        high = torch.maximum(top, x.amax(-1, keepdim=True))
        w, f = torch.exp(x - high), torch.exp(top - high)
        y = (y * f + w @ _from_4_bits(s["v_codes"][slot], s["v_scales"][slot]).permute(0, 2, 1, 3)) / (total * f + w.sum(-1, keepdim=True))
        out[b0:b1] = y.view(n, h_kv, n_q, G, d).permute(0, 2, 1, 3, 4)
    return out[sequence, row].reshape(T, case["h_q"], d).half()


def _run_sparse(s, case):
    """The chosen pages of every row and KV head, and the attention over them."""
    if own:
        cache, batch = s["cache"], (s["table"], s["kv_len"], s["q_start"])
        pages = cache.select(s["q"], s["bounds"], *batch, case["budget"], first=1, recent=2)
        return pages, cache.attention_selected(s["q"], pages, *batch, softcap=case["softcap"])
    page, h_kv, d, T, budget, W = case["page"], case["h_kv"], case["d"], s["T"], case["budget"], s["table"].shape[1]
    G = case["h_q"] // h_kv
    position, _, sequence = _positions(s)
    chosen = _choose(s, case, position, sequence)
    q = s["q"].view(T, h_kv, G, d).float()
    table = s["table"][sequence]                                         # [T, W]
    physical = table[:, None, :].expand(T, h_kv, W).gather(2, chosen.clamp(min=0).long())
    token = torch.arange(page, device=DEVICE)
    key = (chosen[..., None] * page + token).flatten(2)                  # [T, h_kv, budget * page]
    slot = (physical.clamp(min=0).long()[..., None] * page + token).flatten(2)
    head = torch.arange(h_kv, device=DEVICE)[None, :, None]
    x = q @ _from_4_bits(s["k_codes"][slot, head], s["k_scales"][slot, head]).transpose(-1, -2) / math.sqrt(d)
    if case["softcap"]:
        x = case["softcap"] * torch.tanh(x / case["softcap"])
    seen = (key >= 0) & (key <= position[:, None, None]) & (chosen >= 0)[..., None].expand(*chosen.shape, page).flatten(2)
    x = x.masked_fill(~seen[:, :, None, :], -math.inf)
    w = torch.exp(x - x.amax(-1, keepdim=True))
    out = w @ _from_4_bits(s["v_codes"][slot, head], s["v_scales"][slot, head]) / w.sum(-1, keepdim=True)
    return chosen.to(torch.int32), out.reshape(T, case["h_q"], d).half()


def _choose(s, case, position, sequence):
    """The budget pages with the largest bounds on the scores of a KV head's queries, the first and the last two always among them; in order, -1 where there are fewer."""
    page, h_kv, d, T, budget, W = case["page"], case["h_kv"], case["d"], s["T"], case["budget"], s["table"].shape[1]
    bounds, scales = s["bounds"]
    above = torch.zeros(T, h_kv, d, device=DEVICE)
    below = torch.zeros(T, h_kv, d, device=DEVICE)
    for h in range(case["h_q"] // h_kv):                                 # (in this order)
        q = s["q"].view(T, h_kv, -1, d)[:, :, h].float()
        above, below = above + q.clamp(min=0), below + q.clamp(max=0)
    top = torch.maximum(above, -below).amax(-1, keepdim=True)
    r = torch.where(top > 0, torch.full_like(top, 32767.0) / top, 0.0)
    code = torch.round(torch.stack([above, below], 2) * r[..., None]).double().flatten(2)       # [T, h_kv, 2 d] whole numbers
    table = s["table"].long()
    score = torch.empty(T, h_kv, W, device=DEVICE)
    for t in range(T) if W > 4000 else [slice(None)]:
        b = bounds[table[sequence[t]].clamp(min=0)].double().flatten(-2)                        # [.., W, h_kv, 2 d]
        exact_sum = torch.einsum("...hc,...whc->...hw", code[t], b)
        score[t] = exact_sum.float() * scales[table[sequence[t]].clamp(min=0)].transpose(-1, -2)
    column = torch.arange(W, device=DEVICE)
    last = (position // page).clamp(max=W - 1)[:, None, None]
    candidate = (column <= last) & (table[sequence] >= 0)[:, None, :]
    score = torch.where((column < 1) | (column > last - 2), math.inf, score)
    score = torch.where(candidate, score, -math.inf)
    order = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :budget]
    order = torch.where(candidate.expand_as(score).gather(2, order), order, W).sort(-1).values  # (fewer candidates: the others behind)
    order = torch.where(order < W, order, -1)
    return torch.nn.functional.pad(order, (0, budget - order.shape[-1]), value=-1)


# ---------------------------------------------------------------------------- the plain forms' parts
def _positions(s):
    """(position in its sequence, number among the new tokens, sequence) of every row of the call."""
    return _rows_of(s["kv_len"], s["q_start"], s["T"])


def _rows_of(kv_len, q_start, T):
    t = torch.arange(T, device=DEVICE)
    b = torch.searchsorted(q_start[1:], t.to(torch.int32), right=True)
    row = t - q_start[b]
    return kv_len[b] - (q_start[b + 1] - q_start[b]) + row, row, b


def _tokens(s, case, table, kv_len, q_start, T, pool=""):
    """What the cache holds of the last tokens of sequences, keys and values."""
    at, _, b = _rows_of(kv_len, q_start, T)
    slot = table[b, at // case["page"]].clamp(min=0).long() * case["page"] + at % case["page"]
    return tuple(_from_4_bits(s[pool + c + "_codes"][slot], s[pool + c + "_scales"][slot]).half() for c in "kv")


def _to_4_bits(x):
    """x fp16 [..., d] -> (integers [..., d / 32, 32] from -7 to 7, fp16 scales [..., d / 32]): one scale for 32 elements in a row."""
    codes = torch.empty((*x.shape[:-1], x.shape[-1] // GROUP, GROUP), dtype=torch.int8, device=x.device)
    scales = torch.empty(codes.shape[:-1], dtype=torch.float16, device=x.device)
    step = max(1, 2 ** 26 // x[0].numel())
    for i in range(0, x.shape[0], step):
        y = x[i : i + step].float().unflatten(-1, (-1, GROUP))
        scale = (y.abs().amax(-1) / 7.0).half().clamp(max=9352.0)
        code = torch.round(y / scale.float()[..., None]).clamp(-7, 7)
        codes[i : i + step] = torch.where(scale[..., None] == 0, 0.0, code).to(torch.int8)
        scales[i : i + step] = scale
    return codes, scales


def _from_4_bits(code, scale):
    return (code.float() * scale.float()[..., None]).flatten(-2)


# ---------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    page, h_q, h_kv, d = case["page"], case["h_q"], case["h_kv"], case["d"]
    half = h_kv * (d // 2 + d // GROUP * 2)                              # bytes of a token's keys in the cache; its values take the same
    lens = _lengths(case)
    if case["op"] == "fork":
        n = case["children"]
        of = [lens[i * case["parents"] // n] for i in range(n)]
        tables = sum(-(-x // page) * 2 + (x + case["new"]) // page - x // page + 1 for x in of) * 4
        copied = sum(2 * (x % page) * 2 * half for x in of)
        read = sum((x - 1) % page + 1 for x in of) * (2 * half + 4 * h_kv * d)
        return {"bytes": tables + copied + read + 8 * (sum(-(-x // page) for x in lens) + case["spare"]), "flops": 0}
    if case["op"] == "compact":
        # (half of the requests are left; of their pages those behind the last place that the others need move: half, in a pool handed out at random)
        left = sum(lens) - sum(sorted(lens)[: case["B"] // 2])
        pages = sum(-(-n // page) for n in lens)
        return {"bytes": left * (2 * half + 4 * h_kv * d) + left // 2 * 2 * 2 * half + 8 * pages + 12 * (pages + case["spare"]), "flops": 0}
    if case["op"] == "summaries":
        lens, new = _batch(case)
        pages = sum((n - 1) // page - (n - m) // page + 1 for n, m in zip(lens, new))
        read = sum(n - (n - m) // page * page for n, m in zip(lens, new))
        pool = sum(-(-n // page) for n in lens) + 3
        return {"bytes": read * half + 2 * pages * h_kv * (2 * d + 4) + pool * h_kv * 2 * d * 5, "flops": 2 * read * h_kv * d}
    lens, new = _batch(case)
    if case["op"] == "shared":
        kept = case["groups"] * case["prefix"] + sum(lens) - case["B"] * case["prefix"]
        pairs = sum(n - m + i + 1 for n, m in zip(lens, new) for i in range(m))
        return {"bytes": kept * 2 * half + 2 * sum(new) * 2 * h_q * d, "flops": 4 * d * h_q * pairs}
    pages = [min(-(-n // page), case["budget"]) for n in lens]
    looked = sum(-(-n // page) for n in lens) * h_kv * (2 * d + 4)
    tokens = sum(m * min(n, p * page) for n, m, p in zip(lens, new, pages))
    return {"bytes": looked + sum(min(n, m * p * page) for n, m, p in zip(lens, new, pages)) * 2 * half + 2 * sum(new) * 2 * h_q * d + 4 * sum(new) * h_kv * case["budget"],
            "flops": 4 * d * h_q * tokens + sum(m * -(-n // page) for n, m in zip(lens, new)) * h_kv * 4 * d}


# ---------------------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    global own
    kept, own = own, False                                               # (the inputs, and the cache as integers and scales)
    try:
        s = prepare(case, seed)
        return {"fork": _exact_fork, "compact": _exact_compact, "summaries": _exact_summaries, "shared": _exact_shared, "sparse": _exact_sparse}[case["op"]](s, case)
    finally:
        own = kept


def _value(s, c, slot):
    """What the cache stands for at these slots, in 64 bits."""
    x = s[c + "_codes"][slot].double()
    return (x * s[c + "_scales"][slot].double().unsqueeze(-1)).reshape(*x.shape[:-2], -1)


def _exact_fork(s, case):
    """Page by page, as a program on the host would."""
    page, refs, old = case["page"], s["refs"].tolist(), s["table"].tolist()
    parents, lens = s["parents"].tolist(), s["lengths"].tolist()
    table = [[old[p][j] if j * page < n else -1 for j in range(len(old[p]))] for p, n in zip(parents, lens)]
    origin = [list(r) for r in table]                                    # where the tokens of a page came from
    for r in table:
        for x in r:
            if x >= 0:
                refs[x] += 1
    want = [(i, j) for i, n in enumerate(lens) for j in range(n // page, (n + case["new"] - 1) // page + 1) if table[i][j] < 0 or refs[table[i][j]] > 1]
    free = [x for x, n in enumerate(refs) if n == 0]
    missing = max(0, len(want) - len(free))
    if not missing:
        for i, j in want:
            if table[i][j] >= 0:
                refs[table[i][j]] -= 1
        for (i, j), x in zip(want, free):
            table[i][j] = x
            refs[x] += 1
    slot = [origin[i][j // page] * page + j % page for i, n in enumerate(lens) for j in range((n - 1) // page * page, n)]
    slot = torch.tensor(slot, device=DEVICE)
    return _ints(table), _ints(refs), _ints([missing]), _value(s, "k", slot), _value(s, "v", slot)


def _exact_compact(s, case):
    page, refs, table, left = case["page"], s["refs"].tolist(), s["table"].tolist(), s["left"].tolist()
    for b in s["done"].tolist():
        for x in table[b]:
            if x >= 0:
                refs[x] -= 1
        table[b] = [-1] * len(table[b])
    slot = torch.tensor([table[b][j // page] * page + j % page for b, n in enumerate(left) for j in range(n)], dtype=torch.int64, device=DEVICE)
    n = sum(x > 0 for x in refs)
    moved = [x if c > 0 else -1 for x, c in enumerate(refs)]
    holes = [x for x in range(n) if refs[x] == 0]
    for x, to in zip((x for x in range(n, len(refs)) if refs[x] > 0), holes):
        moved[x] = to
    new_refs = [0] * len(refs)
    for x, to in enumerate(moved):
        if to >= 0:
            new_refs[to] = refs[x]
    if slot.numel() * case["h_kv"] * case["d"] > 2 ** 28:
        return _ints([[moved[x] if x >= 0 else -1 for x in r] for r in table]), _ints(new_refs), _ints(moved), None, None
    return _ints([[moved[x] if x >= 0 else -1 for x in r] for r in table]), _ints(new_refs), _ints(moved), _value(s, "k", slot), _value(s, "v", slot)


def _exact_summaries(s, case):
    lens, new = _batch(case)
    page, table = case["page"], s["table"].tolist()
    out = torch.zeros(s["n_pages"], case["h_kv"], 2, case["d"], dtype=torch.float64, device=DEVICE)
    for b, (n, m) in enumerate(zip(lens, new)):
        for j in range((n - m) // page, (n - 1) // page + 1):
            k = _value(s, "k", slice(table[b][j] * page, table[b][j] * page + min(page, n - j * page))).half().double()      # [tokens, h_kv, d]
            top = k.abs().amax((0, 2))
            unit, per = (top / 127).float().double(), torch.where(top > 0, 127 / top, 0.0).float().double()                # (each operation rounded to 32 bits, as defined)
            hi = torch.ceil((k.max(0).values * per[:, None]).float()).clamp(max=127).double()
            lo = torch.floor((k.min(0).values * per[:, None]).float()).clamp(min=-127).double()
            out[table[b][j]] = torch.stack([hi, lo], 1) * unit[:, None, None]
    return out


def _exact_shared(s, case):
    lens, new = _batch(case)
    d, h_q, h_kv, page, table = case["d"], case["h_q"], case["h_kv"], case["page"], s["table"].tolist()
    out = torch.empty(s["T"], h_q, d, dtype=torch.float64, device=DEVICE)
    at = 0
    for b, (n, m) in enumerate(zip(lens, new)):
        slot = torch.tensor([table[b][j // page] * page + j % page for j in range(n)], device=DEVICE)
        k, v = _value(s, "k", slot), _value(s, "v", slot)
        q = s["q"][at : at + m].double().view(m, h_q, d)
        hidden = torch.arange(n, device=DEVICE)[None, :] > torch.arange(n - m, n, device=DEVICE)[:, None]
        for h in range(h_q):
            out[at : at + m, h] = _softmax_of(q[:, h], k[:, h * h_kv // h_q], hidden, case) @ v[:, h * h_kv // h_q]
        at += m
    return out


def _softmax_of(q, k, hidden, case):
    x = torch.einsum("id,jd->ij", q, k) * case["d"] ** -0.5
    if case["softcap"]:
        x = torch.tanh(x / case["softcap"]) * case["softcap"]
    return torch.softmax(x.masked_fill(hidden, -math.inf), -1)


def _exact_sparse(s, case):
    lens, new = _batch(case)
    d, h_q, h_kv, page, table, budget = case["d"], case["h_q"], case["h_kv"], case["page"], s["table"].tolist(), case["budget"]
    G, bounds, scales = h_q // h_kv, *s["bounds"]
    chosen = torch.full((s["T"], h_kv, budget), -1, dtype=torch.int32, device=DEVICE)
    out = torch.empty(s["T"], h_q, d, dtype=torch.float64, device=DEVICE)
    t = 0
    for b, (n, m) in enumerate(zip(lens, new)):
        for p in range(n - m, n):
            here = torch.tensor(table[b][: p // page + 1], device=DEVICE)
            for h in range(h_kv):
                q = s["q"][t].view(h_q, d)[h * G : (h + 1) * G].float()
                up, down = q[0].clamp(min=0), q[0].clamp(max=0)          # sums in 32 bits, head after head, as defined
                for x in q[1:]:
                    up, down = up + x.clamp(min=0), down + x.clamp(max=0)
                top = torch.maximum(up.max(), -down.min()).double()
                per = (32767 / top if top > 0 else top).float().double()
                up, down = (torch.round((x.double() * per).float()).double() for x in (up, down))
                total = bounds[here, h, 0].double() @ up + bounds[here, h, 1].double() @ down
                score = (total.float().double() * scales[here, h].double()).float().tolist()
                ranked = sorted(range(len(score)), key=lambda j: (not (j < 1 or j > len(score) - 3), -score[j], j))
                pages = sorted(ranked[:budget])
                chosen[t, h, : len(pages)] = _ints(pages)
                key = [j * page + i for j in pages for i in range(page) if j * page + i <= p]
                slot = torch.tensor([table[b][j // page] * page + j % page for j in key], device=DEVICE)
                x = s["q"][t].double().view(h_q, d)[h * G : (h + 1) * G]
                k, v = (_value(s, c, (slot, h)) for c in "kv")
                out[t, h * G : (h + 1) * G] = _softmax_of(x, k, torch.zeros(1, len(key), dtype=torch.bool, device=DEVICE), case) @ v
            t += 1
    return chosen, out
