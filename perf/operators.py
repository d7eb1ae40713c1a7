"""The operators of a serving step around the quantised layers: rotary angle tables, keys and values appended to a paged
cache held in 4 bits (with the rotation on the way), attention over that cache, and penalties, biases and masks on the logits.

`own` chooses who computes: the package's kernels, or the plain forms below, elementary torch operations in 32 bits (angles
in 64).  A batch is described the way a serving loop holds it: a page table [sequences, pages], the length of every sequence
with its new tokens (`kv_len`), and where the new tokens of each start in the rows of the call (`q_start`).
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
VOCAB = 128256


def listed():
    return [
        # the angle tables of a model with the frequency scaling of long contexts: up to its first context length, and the whole range
        {"name": "tables_8192_llama3", "op": "tables", "n_pos": 8192, "rot": 128, "base": 500000.0, "scaling": "llama3", "factor": 8.0},
        {"name": "tables_131072_yarn", "op": "tables", "n_pos": 131072, "rot": 128, "base": 10000.0, "scaling": "yarn", "factor": 16.0},
        # one user's generated token goes to the cache, at the length of the 1024 + 256 token protocol
        {"name": "append_token", "op": "append", "B": 1, "longest": 1280, "shortest": 1280, "new": 1, "mix": 0, "page": 16, "rot": 128, "interleaved": False, **LLAMA31_8B},
        # ragged prompts of one step, 8 requests: the cache is filled
        {"name": "append_prompts", "op": "append", "B": 8, "longest": 2048, "shortest": 300, "new": 0, "mix": 3, "page": 64, "rot": 128, "interleaved": False, **LLAMA31_8B},
        # one user: a generated token at 1280 positions, and at the end of a long document
        {"name": "decode_1_at_1280", "op": "attention", "B": 1, "longest": 1280, "shortest": 1280, "new": 1, "mix": 0, "page": 16, "window": 0, "softcap": 0.0, **LLAMA31_8B},
        {"name": "decode_1_at_131071", "op": "attention", "B": 1, "longest": 131071, "shortest": 131071, "new": 1, "mix": 0, "page": 64, "window": 0, "softcap": 0.0, **LLAMA31_8B},
        # a serving batch of ragged lengths, small pages
        {"name": "decode_64_ragged", "op": "attention", "B": 64, "longest": 8192, "shortest": 500, "new": 1, "mix": 5, "page": 16, "window": 0, "softcap": 0.0, **LLAMA31_8B},
        # the same with wide heads, a sliding window and a soft cap on the scores
        {"name": "decode_24_window", "op": "attention", "B": 24, "longest": 7001, "shortest": 900, "new": 1, "mix": 9, "page": 32, "window": 4096, "softcap": 50.0, **GEMMA2_2B},
        # ragged prompts attend to themselves
        {"name": "prompts_3_of_4096", "op": "attention", "B": 3, "longest": 4096, "shortest": 1000, "new": 0, "mix": 2, "page": 64, "window": 0, "softcap": 0.0, **LLAMA31_8B},
        # a chunk of a long prompt, over what is cached of it
        {"name": "chunk_512_at_16384", "op": "attention", "B": 1, "longest": 16384, "shortest": 16384, "new": 512, "mix": 0, "page": 64, "window": 0, "softcap": 0.0, **LLAMA31_8B},
        # one request's logits under a grammar, and a batch's
        {"name": "logits_1", "op": "logits", "rows": 1, "vocab": VOCAB, "history": 1280, "mix": 0, "biases": 32, "mask": True, "dtype": "fp16"},
        {"name": "logits_256", "op": "logits", "rows": 256, "vocab": VOCAB, "history": 4096, "mix": 4, "biases": 300, "mask": True, "dtype": "fp16"},
    ]


def _log_int(rng, lo, hi, step=1):
    return max(step, round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step) * step)


def draw(rng):
    op = rng.choice(["tables", "append", "attention", "attention", "attention", "logits"])
    if op == "tables":
        rot = rng.choice([32, 64, 128, 256])
        return {"op": op, "n_pos": _log_int(rng, 500, 131072 * 128 // rot), "rot": rot, "base": rng.choice([10000.0, 500000.0]),
                "scaling": rng.choice(["none", "linear", "ntk", "llama3", "yarn"]), "factor": rng.choice([2.0, 4.0, 8.0, 16.0])}
    if op == "logits":
        vocab = rng.choice([VOCAB, 256000, 50257, 32001, _log_int(rng, 1000, 130000)])
        return {"op": op, "rows": _log_int(rng, 1, 256 * VOCAB // max(vocab, VOCAB)), "vocab": vocab, "history": _log_int(rng, 4, 8192), "mix": rng.randrange(1 << 20),
                "biases": rng.choice([0, 7, 300]), "mask": rng.random() < 0.7, "dtype": rng.choice(["fp16", "fp16", "fp32"])}
    heads = rng.choice([LLAMA31_8B, LLAMA31_8B, GEMMA2_2B, {"h_q": 14, "h_kv": 2, "d": 64}, {"h_q": 16, "h_kv": 16, "d": 64}, {"h_q": 12, "h_kv": 1, "d": 128}])
    page, mix = rng.choice([16, 32, 64, 128]), rng.randrange(1 << 20)
    wide = heads["h_kv"] * heads["d"]
    if op == "append":
        longest = _log_int(rng, 1, 4096)
        most = max(1, 8 * 2048 * 1024 // (longest * wide))
        return {"op": op, "B": _log_int(rng, 1, max(1, min(256, most))), "longest": longest, "shortest": max(1, longest // 3), "new": rng.choice([0, 1, 1, 5]), "mix": mix, "page": page,
                "rot": rng.choice([heads["d"], heads["d"], heads["d"] // 2, 32]), "interleaved": rng.random() < 0.4, **heads}
    case = {"op": op, "mix": mix, "page": page, "window": rng.choice([0, 0, 0, 100, 4096]), "softcap": rng.choice([0.0, 0.0, 0.0, 50.0]), **heads}
    kind = rng.choice(["token", "token", "few", "chunk", "prompt"])
    if kind in ("token", "few"):
        longest = _log_int(rng, 10, 100000)
        most = max(1, min(256, 64 * 8192 * 1024 // (longest * wide)))
        return {**case, "B": _log_int(rng, 1, most), "longest": longest, "shortest": max(1, longest // rng.choice([1, 4, 16])), "new": 1 if kind == "token" else rng.randint(2, 6)}
    if kind == "chunk":
        new = _log_int(rng, 20, 700)
        longest = new + _log_int(rng, 10, 512 * 16384 // new * 32 // (heads["h_q"] + 16))
        longest = min(longest, 60000)
        return {**case, "B": 1, "longest": longest, "shortest": longest, "new": new}
    longest = _log_int(rng, 30, 3500)
    most = max(1, 2 * 3500 * 3500 // (longest * longest))
    return {**case, "B": _log_int(rng, 1, min(24, most)), "longest": longest, "shortest": max(1, longest // 3), "new": 0}


# ---------------------------------------------------------------------------- what a case holds
def _lengths(case):
    """(length with the new tokens, new tokens) of every sequence: the first is the longest, the others are spread over the logarithm."""
    rng = random.Random(case["mix"])
    lens = [case["longest"]] + [_log_int(rng, case["shortest"], case["longest"]) for _ in range(case["B"] - 1)]
    return lens, [n if case["new"] == 0 else min(case["new"], n) for n in lens]


def _history(case):
    """(tokens of the history, tokens of it that are the prompt) of every row."""
    rng = random.Random(case["mix"])
    lens = [case["history"]] + [_log_int(rng, max(1, case["history"] // 8), case["history"]) for _ in range(case["rows"] - 1)]
    return lens, [n * 4 // 5 for n in lens]


def _starts(counts):
    return [sum(counts[:i]) for i in range(len(counts) + 1)]


def _generator(seed):
    return torch.Generator(device=DEVICE).manual_seed(seed)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEVICE)


def prepare(case, seed):
    g = _generator(seed)
    if case["op"] == "tables":                                           # (the first position is the input: a table that continues another)
        return {"case": case, "first": random.Random(seed).randrange(1000)}
    return _prepare_logits(case, g) if case["op"] == "logits" else _prepare_cache(case, g)


def _prepare_cache(case, g):
    lens, new = _lengths(case)
    B, page, h_q, h_kv, d = case["B"], case["page"], case["h_q"], case["h_kv"], case["d"]
    T, widest = sum(new), max(-(-n // page) for n in lens)
    n_pages = sum(-(-n // page) for n in lens) + 3
    s = {"case": case, "kv_len": _ints(lens), "q_start": _ints(_starts(new)), "max_q": max(new), "T": T}
    # pages in the order in which a busy pool would hand them out; entries behind a sequence's last page hold nothing
    order = torch.randperm(n_pages, generator=g, device=DEVICE).to(torch.int32)
    used = torch.arange(widest, device=DEVICE)[None, :] < ((s["kv_len"] + page - 1) // page)[:, None]
    table = torch.full((B, widest), -1, dtype=torch.int32, device=DEVICE)
    table[used] = order[: n_pages - 3]
    s["table"] = table
    s["q"] = torch.randn(T, h_q * d, generator=g, device=DEVICE, dtype=torch.float16)
    # keys of a trained model: some channels of a head are several times larger than the others
    channel = torch.exp(0.5 * torch.randn(h_kv * d, generator=g, device=DEVICE)).half()
    if case["op"] == "append":
        s["k"] = torch.randn(T, h_kv * d, generator=g, device=DEVICE, dtype=torch.float16) * channel
        s["v"] = torch.randn(T, h_kv * d, generator=g, device=DEVICE, dtype=torch.float16)
        angle = torch.outer(torch.arange(max(lens), device=DEVICE, dtype=torch.float64), _frequencies(case["rot"], 500000.0, "none", 1.0).to(DEVICE))
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
        if own:
            s["cache"] = _package().PagedKV(n_pages, page, h_kv, d, device=DEVICE)
        return s
    # attention: a pool that is full
    slots = n_pages * page
    k = torch.randn(slots, h_kv * d, generator=g, device=DEVICE, dtype=torch.float16) * channel
    v = torch.randn(slots, h_kv * d, generator=g, device=DEVICE, dtype=torch.float16)
    if own:
        s["cache"] = _package().PagedKV(n_pages, page, h_kv, d, device=DEVICE)
        s["cache"].append(k, v, torch.arange(n_pages, dtype=torch.int32, device=DEVICE)[None, :], _ints([slots]), _ints([0, slots]))
    else:
        s["k_codes"], s["k_scales"] = _to_4_bits(k.view(slots, h_kv, d))
        s["v_codes"], s["v_scales"] = _to_4_bits(v.view(slots, h_kv, d))
    return s


def _prepare_logits(case, g):
    R, V = case["rows"], case["vocab"]
    lens, prompt = _history(case)
    n = sum(lens)
    s = {"case": case, "start": _ints(_starts(lens)), "n_prompt": _ints(prompt)}
    s["logits"] = (3.0 * torch.randn(R, V, generator=g, device=DEVICE)).to(torch.float16 if case["dtype"] == "fp16" else torch.float32)
    # text repeats itself: few tokens are frequent
    s["tokens"] = (V * torch.rand(n, generator=g, device=DEVICE) ** 4).to(torch.int32).clamp_(max=V - 1)
    s["repetition"] = 1.0 + 0.3 * torch.rand(R, generator=g, device=DEVICE)
    s["presence"] = 0.5 * torch.rand(R, generator=g, device=DEVICE)
    s["frequency"] = 0.2 * torch.rand(R, generator=g, device=DEVICE)
    nb = min(case["biases"], V)
    if nb:                                                               # (a row lists a token once)
        first = torch.randint(0, V, (R, 1), generator=g, device=DEVICE)
        s["bias_ids"] = ((first + (V // nb) * torch.arange(nb, device=DEVICE)[None, :]) % V).to(torch.int32).reshape(-1)
        s["bias_values"] = 5.0 * torch.randn(R * nb, generator=g, device=DEVICE)
        s["bias_start"] = _ints([nb * i for i in range(R + 1)])
    if case["mask"]:                                                     # a grammar allows about one token in four
        words = (R, (V + 31) // 32)
        a, b = (torch.randint(-(1 << 31), 1 << 31, words, generator=g, device=DEVICE, dtype=torch.int64).to(torch.int32) for _ in range(2))
        s["mask"] = a & b
    return s


# ---------------------------------------------------------------------------- one pass
def _package():
    import paper_2505_00232_b200
    return paper_2505_00232_b200


def run(s):
    case = s["case"]
    return {"tables": _run_tables, "append": _run_append, "attention": _run_attention, "logits": _run_logits}[case["op"]](s, case)


def _run_tables(s, case):
    if own:
        return _package().qlinear_rope_tables(case["n_pos"], case["rot"], case["base"], scaling=None if case["scaling"] == "none" else case["scaling"], factor=case["factor"], original=8192,
                                              first=s["first"], device=DEVICE)
    f = _frequencies(case["rot"], case["base"], case["scaling"], case["factor"]).to(DEVICE)
    angle = torch.outer(torch.arange(s["first"], s["first"] + case["n_pos"], device=DEVICE, dtype=torch.float64), f)
    m = _magnitude(case["scaling"], case["factor"])
    return (angle.cos() * m).float(), (angle.sin() * m).float()


def _run_append(s, case):
    """The rotated queries, and what the cache then stands for at the places of the new tokens."""
    batch = (s["table"], s["kv_len"], s["q_start"])
    if own:
        q = s["cache"].append(s["k"], s["v"], *batch, q=s["q"], cos=s["cos"], sin=s["sin"], interleaved=case["interleaved"])
        k, v = s["cache"].read(*batch, s["T"])
        return q, k, v
    h_q, h_kv, d, T = case["h_q"], case["h_kv"], case["d"], s["T"]
    at = _positions(s)[0]
    q = _rotated(s["q"].view(T, h_q, d), s["cos"][at], s["sin"][at], case["rot"], case["interleaved"])
    k = _rotated(s["k"].view(T, h_kv, d), s["cos"][at], s["sin"][at], case["rot"], case["interleaved"])
    return q.view(T, h_q * d), _from_4_bits(*_to_4_bits(k)).half(), _from_4_bits(*_to_4_bits(s["v"].view(T, h_kv, d))).half()


def _run_attention(s, case):
    if own:
        return s["cache"].attention(s["q"], s["table"], s["kv_len"], s["q_start"], s["max_q"], softcap=case["softcap"], window=case["window"])
    B, page, h_kv, d, T, n_q = case["B"], case["page"], case["h_kv"], case["d"], s["T"], s["max_q"]
    group = case["h_q"] // h_kv
    L = s["table"].shape[1] * page
    key = torch.arange(L, device=DEVICE)
    slot = (s["table"].clamp(min=0).long() * page)[:, key // page] + key % page              # [B, L]
    position, row, sequence = _positions(s)
    q = torch.zeros(B, n_q, h_kv, group, d, device=DEVICE)
    q[sequence, row] = s["q"].view(T, h_kv, group, d).float()
    at = torch.full((B, n_q), -1, device=DEVICE)
    at[sequence, row] = position
    q = q.permute(0, 2, 1, 3, 4).reshape(B, h_kv, n_q * group, d)
    score = q @ _from_4_bits(s["k_codes"][slot], s["k_scales"][slot]).permute(0, 2, 3, 1) / math.sqrt(d)
    if case["softcap"]:
        score = case["softcap"] * torch.tanh(score / case["softcap"])
    seen = key[None, None, :] <= at[:, :, None]
    if case["window"]:
        seen &= key[None, None, :] > at[:, :, None] - case["window"]
    score = score.view(B, h_kv, n_q, group, L).masked_fill_(~seen[:, None, :, None, :], -math.inf)
    weight = torch.exp(score - score.amax(-1, keepdim=True).clamp(min=-1e30))
    weight /= weight.sum(-1, keepdim=True).clamp(min=1e-30)
    out = weight.view(B, h_kv, n_q * group, L) @ _from_4_bits(s["v_codes"][slot], s["v_scales"][slot]).permute(0, 2, 1, 3)
    out = out.view(B, h_kv, n_q, group, d).permute(0, 2, 1, 3, 4)[sequence, row]
    return out.reshape(T, case["h_q"], d).half()


def _run_logits(s, case):
    if own:
        return _package().qlinear_adjust_logits(s["logits"], s["tokens"], s["start"], s["n_prompt"], repetition=s["repetition"], presence=s["presence"], frequency=s["frequency"],
                                                bias_ids=s.get("bias_ids"), bias_values=s.get("bias_values"), bias_start=s.get("bias_start"), mask=s.get("mask"))
    R, V = case["rows"], case["vocab"]
    n = s["tokens"].numel()
    i = torch.arange(n, device=DEVICE)
    row = torch.searchsorted(s["start"][1:], i.to(torch.int32), right=True)
    place = row * V + s["tokens"].long()
    output = (i - s["start"][row] >= s["n_prompt"][row]).to(torch.int32)
    seen = torch.zeros(R * V, dtype=torch.bool, device=DEVICE).index_fill_(0, place, True).view(R, V)
    count = torch.zeros(R * V, dtype=torch.int32, device=DEVICE).index_add_(0, place, output).view(R, V)
    x = s["logits"].float()
    r = s["repetition"][:, None]
    x = torch.where(seen, torch.where(x > 0, x / r, x * r), x)
    x = x - s["frequency"][:, None] * count - s["presence"][:, None] * (count > 0)
    if "bias_ids" in s:
        where = torch.searchsorted(s["bias_start"][1:], torch.arange(s["bias_ids"].numel(), device=DEVICE, dtype=torch.int32), right=True) * V + s["bias_ids"].long()
        x = x.reshape(-1).index_add_(0, where, s["bias_values"]).view(R, V)
    if "mask" in s:
        token = torch.arange(V, device=DEVICE)
        x = torch.where((s["mask"][:, token // 32] >> (token % 32)) & 1 == 1, x, -math.inf)
    return x.to(s["logits"].dtype)


# ---------------------------------------------------------------------------- the plain forms' parts
def _frequencies(rot, base, scaling, factor, original=8192):
    """Radians per position of the rot / 2 pairs, in 64 bits."""
    i = torch.arange(rot // 2, dtype=torch.float64)
    if scaling == "ntk":                                                 # the base that leaves the fastest pair as it is and slows the slowest by the factor
        base = base * factor ** (rot / (rot - 2))
    f = base ** (-2 * i / rot)
    if scaling == "linear":
        return f / factor
    if scaling == "llama3":                                              # pairs that turn more than 4 times within the first length stay, under once are slowed, smooth between
        smooth = ((original * f / (2 * math.pi) - 1.0) / (4.0 - 1.0)).clamp(0, 1)
        return f / factor * (1 - smooth) + f * smooth
    if scaling == "yarn":                                                # the same by the pair's number: a ramp between the pairs that turn 32 times and once
        at = lambda turns: rot * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(base))
        low, high = max(math.floor(at(32.0)), 0), min(math.ceil(at(1.0)), rot - 1)
        ramp = ((i - low) / max(high - low, 0.001)).clamp(0, 1)
        return f / factor * ramp + f * (1 - ramp)
    return f


def _magnitude(scaling, factor):
    return 0.1 * math.log(factor) + 1.0 if scaling == "yarn" else 1.0


def _positions(s):
    """(position in its sequence, number among the new tokens, sequence) of every row of the call."""
    t = torch.arange(s["T"], device=DEVICE)
    b = torch.searchsorted(s["q_start"][1:], t.to(torch.int32), right=True)
    row = t - s["q_start"][b]
    return s["kv_len"][b] - (s["q_start"][b + 1] - s["q_start"][b]) + row, row, b


def _rotated(x, cos, sin, rot, interleaved):
    """x fp16 [T, heads, d]: its first `rot` elements turned, in pairs of neighbours or of the two halves."""
    c, s = cos[:, None, : rot // 2], sin[:, None, : rot // 2]
    y = x.clone()
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., : rot // 2], x[..., rot // 2 : rot])
    first, second = a.float() * c - b.float() * s, b.float() * c + a.float() * s
    if interleaved:
        y[..., 0:rot:2], y[..., 1:rot:2] = first.half(), second.half()
    else:
        y[..., : rot // 2], y[..., rot // 2 : rot] = first.half(), second.half()
    return y


def _to_4_bits(x):
    """x fp16 [..., d] -> (integers [..., d / 32, 32] from -7 to 7, fp16 scales [..., d / 32]): one scale for 32 elements in a row."""
    x = x.float().unflatten(-1, (-1, GROUP))
    scale = (x.abs().amax(-1) / 7.0).half().clamp(max=9352.0)
    code = torch.round(x / scale.float()[..., None]).clamp(-7, 7)
    return torch.where(scale[..., None] == 0, 0.0, code).to(torch.int8), scale


def _from_4_bits(code, scale):
    return (code.float() * scale.float()[..., None]).flatten(-2)


# ---------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    if case["op"] == "tables":
        return {"bytes": 2 * case["n_pos"] * (case["rot"] // 2) * 4, "flops": case["n_pos"] * case["rot"] // 2}
    if case["op"] == "logits":
        lens, _ = _history(case)
        n = case["rows"] * case["vocab"]
        size = 2 if case["dtype"] == "fp16" else 4
        return {"bytes": 2 * size * n + 4 * sum(lens) + 8 * case["rows"] * case["biases"] + (n // 8 if case["mask"] else 0), "flops": n}
    lens, new = _lengths(case)
    h_q, h_kv, d = case["h_q"], case["h_kv"], case["d"]
    kept = 2 * h_kv * (d // 2 + d // GROUP * 2)                          # bytes of a token in the cache
    if case["op"] == "append":
        T = sum(new)
        return {"bytes": T * (2 * (h_q + 2 * h_kv) * d + 4 * case["rot"] + 2 * h_q * d + kept + 2 * 2 * h_kv * d), "flops": 3 * T * (h_q + h_kv) * case["rot"]}
    window = case["window"] or max(lens)
    pairs = sum(min(n - m + i + 1, window) for n, m in zip(lens, new) for i in range(m))
    read = sum(min(n, m - 1 + window) for n, m in zip(lens, new))
    return {"bytes": read * kept + 2 * sum(new) * 2 * h_q * d, "flops": 4 * d * h_q * pairs}


# ---------------------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    global own
    kept, own = own, False                                               # (the inputs, and the cache as integers and scales)
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    return {"tables": _exact_tables, "append": _exact_append, "attention": _exact_attention, "logits": _exact_logits}[case["op"]](s, case)


def _exact_tables(s, case):
    # turns of every pair per position, reduced to the fraction of a turn before it becomes an angle
    rot, base, factor = case["rot"], case["base"], case["factor"]
    turns = []
    for i in range(rot // 2):
        b = base * factor ** (rot / (rot - 2)) if case["scaling"] == "ntk" else base
        f = math.exp(-2 * i / rot * math.log(b))
        if case["scaling"] == "linear":
            f /= factor
        if case["scaling"] == "llama3":
            cycles = 8192 * f / (2 * math.pi)
            f = f if cycles >= 4 else f / factor if cycles <= 1 else f * ((cycles - 1) / 3 + (4 - cycles) / 3 / factor)
        if case["scaling"] == "yarn":
            low = max(math.floor(rot / 2 * math.log(8192 / (64 * math.pi), base)), 0)
            high = min(math.ceil(rot / 2 * math.log(8192 / (2 * math.pi), base)), rot - 1)
            part = min(max((i - low) / max(high - low, 0.001), 0.0), 1.0)
            f *= 1 - part + part / factor
        turns.append(f / (2 * math.pi))
    x = torch.arange(s["first"], s["first"] + case["n_pos"], device=DEVICE, dtype=torch.float64)[:, None] * torch.tensor(turns, dtype=torch.float64, device=DEVICE)
    x = 2 * math.pi * (x - torch.round(x))
    m = 1 + math.log(factor) / 10 if case["scaling"] == "yarn" else 1
    return m * torch.cos(x), m * torch.sin(x)


def _exact_append(s, case):
    d, rot = case["d"], case["rot"]
    q0, starts, lens = 0, s["q_start"].tolist(), s["kv_len"].tolist()
    at = torch.cat([torch.arange(n - (starts[b + 1] - starts[b]), n) for b, n in enumerate(lens)]).to(DEVICE)
    turn = torch.complex(s["cos"][at].double(), s["sin"][at].double())[:, None, :]

    def rotated(x):                                                      # pairs as complex numbers; stored as fp16
        x = x.view(x.shape[0], -1, d).double()
        head, rest = x[..., :rot], x[..., rot:]
        pair = head.unflatten(-1, (-1, 2)) if case["interleaved"] else head.unflatten(-1, (2, -1)).transpose(-1, -2)
        y = torch.view_as_real(torch.complex(pair[..., 0].contiguous(), pair[..., 1].contiguous()) * turn)
        y = y.flatten(-2) if case["interleaved"] else y.transpose(-1, -2).flatten(-2)
        return torch.cat([y, rest], -1).half().double()

    def held(x):                                                         # what 4 bits and a scale for 32 elements keep
        x = x.view(x.shape[0], -1, d // 32, 32)
        scale = (x.abs().max(-1, keepdim=True).values / 7).half().double().clamp(max=9352)
        return torch.where(scale > 0, scale * torch.clamp(torch.round(x / scale), -7, 7), 0.0).flatten(-2)

    q, k = rotated(s["q"]), rotated(s["k"])
    return q.flatten(1), held(k), held(s["v"].view(-1, case["h_kv"], d).double())


def _exact_attention(s, case):
    if sum(n * m for n, m in zip(*_lengths(case))) * case["h_q"] * case["d"] > 1e12:
        return None
    d, h_q, h_kv, page = case["d"], case["h_q"], case["h_kv"], case["page"]
    starts, lens, table = s["q_start"].tolist(), s["kv_len"].tolist(), s["table"].tolist()
    out = torch.empty(s["T"], h_q, d, dtype=torch.float64, device=DEVICE)
    for b, n in enumerate(lens):
        slot = torch.tensor([table[b][j // page] * page + j % page for j in range(n)], device=DEVICE)
        k, v = ((s[c + "_codes"][slot].double() * s[c + "_scales"][slot].double()[..., None]).flatten(2) for c in "kv")
        q = s["q"][starts[b] : starts[b + 1]].double().view(-1, h_q, d)
        m = q.shape[0]
        i, j = torch.arange(n - m, n, device=DEVICE)[:, None], torch.arange(n, device=DEVICE)[None, :]
        hidden = (j > i) | (i - j >= (case["window"] or n + 1))
        for h in range(h_q):
            x = torch.einsum("id,jd->ij", q[:, h], k[:, h * h_kv // h_q]) * d ** -0.5
            if case["softcap"]:
                x = torch.tanh(x / case["softcap"]) * case["softcap"]
            out[starts[b] : starts[b + 1], h] = torch.softmax(x.masked_fill(hidden, -math.inf), -1) @ v[:, h * h_kv // h_q]
    return out


def _exact_logits(s, case):
    x, starts, prompt = s["logits"].double(), s["start"].tolist(), s["n_prompt"].tolist()
    for r in range(case["rows"]):
        tokens = s["tokens"][starts[r] : starts[r + 1]].long()
        seen = torch.unique(tokens)
        said, times = torch.unique(tokens[prompt[r] :], return_counts=True)
        rep = s["repetition"][r].double()
        x[r, seen] = torch.where(x[r, seen] > 0, x[r, seen] / rep, x[r, seen] * rep)
        x[r, said] -= s["presence"][r].double() + s["frequency"][r].double() * times
        if "bias_ids" in s:
            n = s["bias_ids"].numel() // case["rows"]
            x[r, s["bias_ids"][n * r : n * r + n].long()] += s["bias_values"][n * r : n * r + n].double()
        if "mask" in s:
            bits = (s["mask"][r].view(torch.uint8)[:, None] >> torch.arange(8, device=DEVICE, dtype=torch.uint8)) & 1
            x[r, bits.flatten()[: case["vocab"]] == 0] = -math.inf
    return x
