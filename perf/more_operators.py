"""Operators over a paged cache of keys and values held in 8 bits, as cases for timing and comparison.

A case is a dict of plain values; `op` names the public entry point:

  append   amd.append_fp8: rotates the new rows' q and k, rounds k and v to e4m3 with a scale for each page of 64 tokens and
           head, and stores them as the last entries of their sequences
  attend   amd.attend_fp8: causal attention of the last rows over the cache, whole or with a sliding window and a few first
           tokens that stay visible
  weigh    amd.weigh_fp8: adds the attention weight that every entry got from these rows to what it has got so far
  evict    amd.evict_fp8: keeps the first tokens, the last ones and, of those between, the ones of the largest weight, for each
           head, and moves them into pages of their own

Heads are those of synth.config's models (queries over keys), lengths its prompts and beyond.  The plain forms are elementary
torch operations; `exact` is the definition in 64 bits, written apart from them.
"""
from __future__ import annotations

import math
import random

import torch

own = False

PAGE = 64                    # tokens of a page, which share a scale in each head
E4M3 = torch.float8_e4m3fn
LEAST = -100                 # the least exponent of a scale
BF16 = torch.bfloat16


def listed():
    def case(name, op, heads, kv, d, seqs, rows, length, **more):
        return {"name": name, "op": op, "heads": heads, "kv": kv, "d": d, "seqs": seqs, "rows": rows, "len": length, **more}

    return [
        # one token of the 70B shape behind a 4096-token prompt: all latency
        case("append_64over8_m1", "append", 64, 8, 128, 1, 1, 4097, ragged=False, theta=10000.0),
        # that prompt itself
        case("append_64over8_m4095", "append", 64, 8, 128, 1, 4095, 4095, ragged=False, theta=10000.0),
        # a decode step of the 70B shape behind its prompt
        case("attend_64over8_m1", "attend", 64, 8, 128, 1, 1, 4097, ragged=False, window=0, sinks=0),
        # a verify window of 7 and its bonus row behind a long text
        case("attend_64over8_m8_long", "attend", 64, 8, 128, 1, 8, 131072, ragged=False, window=0, sinks=0),
        # decode of 16 requests of the 7B shape, all of different lengths
        case("attend_32over32_b16_m1", "attend", 32, 32, 128, 16, 1, 8192, ragged=True, window=0, sinks=0),
        # verify windows of several requests that see their first 4 tokens and the last 1024
        case("attend_64over8_b8_m8_window", "attend", 64, 8, 128, 8, 8, 32768, ragged=True, window=1024, sinks=4),
        # the 70B shape's prompt
        case("attend_64over8_m4095", "attend", 64, 8, 128, 1, 4095, 4095, ragged=False, window=0, sinks=0),
        # a chunk of a longer prompt through the 1B draft model, with a window
        case("attend_32over4_m2047_window", "attend", 32, 4, 64, 1, 2047, 6143, ragged=False, window=1000, sinks=4),
        # what a decode step of 8 requests adds to the weights
        case("weigh_64over8_b8_m1", "weigh", 64, 8, 128, 8, 1, 8192, ragged=True, window=0, sinks=0),
        # the weights of a 2047-token prompt
        case("weigh_64over8_m2047", "weigh", 64, 8, 128, 1, 2047, 2047, ragged=False, window=0, sinks=0),
        # one request of the small pair whose cache has become too long
        case("evict_16over16", "evict", 16, 16, 128, 1, 1, 4096, ragged=False, budget=1024, sinks=4, recent=256),
        # 16 requests of the 70B shape at once
        case("evict_64over8_b16", "evict", 64, 8, 128, 16, 1, 16384, ragged=True, budget=2048, sinks=4, recent=500),
    ]


HEADS = [(4, 4, 64), (16, 16, 128), (32, 32, 128), (32, 4, 64), (56, 56, 128), (64, 8, 128)]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "attend", "weigh", "evict"])
    heads, kv, d = rng.choice(HEADS)
    seqs = rng.choice([1, _log_int(rng, 1, 32)])
    length = _log_int(rng, 1, min(131072, (1 << 28) // (seqs * kv * d)))
    rows = min(length, rng.choice([1, rng.randint(2, 17), _log_int(rng, 17, 4096)]))
    rows = max(1, min(rows, (1 << 29) // (seqs * heads * length), 16384 // seqs))
    case = {"op": op, "heads": heads, "kv": kv, "d": d, "seqs": seqs, "rows": rows, "len": length, "ragged": rng.choice([False, True])}
    if op == "append":
        case["theta"] = rng.choice([0.0, 10000.0, 500000.0])
    elif op == "evict":
        case["rows"] = 1
        case["budget"] = max(1, _log_int(rng, max(1, length // 16), length + 100))
        case["sinks"] = min(rng.choice([0, 4]), case["budget"])
        case["recent"] = rng.randint(0, case["budget"] - case["sinks"])
    else:
        case["window"] = rng.choice([0, 0, _log_int(rng, 1, length + 1)])
        case["sinks"] = rng.choice([0, 4, rng.randint(1, 100)]) if case["window"] else 0
    return case


# ---- inputs ----------------------------------------------------------------------------------
def _sizes(case):
    """(rows, length) of every sequence, from the case alone."""
    if not case["ragged"]:
        return [(case["rows"], case["len"])] * case["seqs"]
    rng = random.Random(case["seqs"] * 1000003 + case["len"] * 101 + case["rows"])
    got = []
    for i in range(case["seqs"]):
        rows = case["rows"] if i == 0 else rng.randint(1, case["rows"])
        got.append((rows, case["len"] if i == 0 else rng.randint(max(rows, case["len"] // 8), case["len"])))
    return got


def _pages(n):
    return -(-n // PAGE)


def _exponent(top):
    """The least e of 448 * 2^e >= top, and not below LEAST."""
    m, x = torch.frexp(top)
    return torch.where(m <= 0.875, x - 9, x - 8).clamp_min(LEAST)


def _power(e):
    """2^e in fp32; below its normal numbers, where a code comes to nothing, their least."""
    return ((e.clamp_min(-126) + 127).to(torch.int32) << 23).view(torch.float32)


def _token_codes(x):
    """e4m3 codes (as bytes) of pages [...][tokens][d] and their exponents [...]."""
    e = _exponent(x.abs().amax(dim=(-1, -2)))
    return (x * _power(-e)[..., None, None]).to(E4M3).view(torch.uint8), e


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda")
    heads, kv, d = case["heads"], case["kv"], case["d"]
    sizes = _sizes(case)
    width = max(_pages(n) for _, n in sizes) + 1
    spare = sum(_pages(n) for _, n in sizes) + 5
    ids = torch.randperm(spare, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(sizes), width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, (_, n) in enumerate(sizes):
        table[i, : _pages(n)] = ids[at : at + _pages(n)]
        at += _pages(n)
    # keys with a few channels above the rest, values without; a page's level differs from the next one's
    channels = torch.where(torch.rand(d, generator=g, device="cuda") < 0.05, 4.0, 1.0)
    codes, scale = [], []
    for level in (channels, torch.ones(d, device="cuda")):
        pool, e = torch.empty(spare, kv, PAGE, d, dtype=torch.uint8, device="cuda"), []
        for i in range(0, spare, 1024):                     # so many pages at a time in fp32
            x = normal(min(1024, spare - i), kv, PAGE, d) * level
            part, low = _token_codes(x * torch.exp(0.3 * normal(x.shape[0], kv, 1, 1)))
            pool[i : i + x.shape[0]] = part
            e.append(low)
        codes.append(pool)
        scale.append(_power(torch.cat(e)))
    s = {"k": codes[0].view(E4M3), "v": codes[1].transpose(2, 3).contiguous().view(E4M3), "scale": torch.stack(scale, 2), "table": table}
    s["len"] = torch.tensor([n for _, n in sizes], dtype=torch.int32, device="cuda")
    starts = [0]
    for m, _ in sizes:
        starts.append(starts[-1] + m)
    s["rows"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
    s["most"] = max(m for m, _ in sizes)                    # rows of the longest sequence, for the plain form's padding
    n = starts[-1]
    if case["op"] == "append":
        # slices of one QKV projection
        qkv = normal(n, (heads + 2 * kv) * d).to(BF16)
        s["q"] = qkv[:, : heads * d].view(n, heads, d)
        s["new_k"] = qkv[:, heads * d : (heads + kv) * d].view(n, kv, d)
        s["new_v"] = qkv[:, (heads + kv) * d :].view(n, kv, d)
    elif case["op"] == "evict":
        # weights as attention leaves them: most next to nothing, some heavy, equal ones among them
        w = torch.exp(2.5 * normal(len(sizes), kv, width * PAGE) - 4)
        s["weight"] = torch.where(w < 0.002, 0.0, w)
        fresh = _pages(case["budget"])
        s["to_table"] = torch.randperm(len(sizes) * fresh, generator=g, device="cuda").to(torch.int32).view(len(sizes), fresh)
        shape = (len(sizes) * fresh, kv)
        s["to_k"] = torch.zeros(*shape, PAGE, d, dtype=torch.uint8, device="cuda").view(E4M3)
        s["to_v"] = torch.zeros(*shape, d, PAGE, dtype=torch.uint8, device="cuda").view(E4M3)
        s["to_scale"] = torch.zeros(*shape, 2, device="cuda")
        s["to_len"] = torch.zeros(len(sizes), dtype=torch.int32, device="cuda")
        s["to_weight"] = torch.zeros(len(sizes), kv, fresh * PAGE, device="cuda")
    else:
        s["q"] = normal(n, heads, d).to(BF16)
    if case["op"] == "weigh":
        s["weight"] = torch.rand(len(sizes), kv, width * PAGE, generator=g, device="cuda")
        s["lse"] = math.log(case["len"]) + 0.6 + 0.3 * normal(n, heads)        # an input like any other
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        import paper_2408_11850_amd as amd

        s["amd"] = amd
        amd.load_library()
        s["cache"] = amd.Fp8Cache(s["k"], s["v"], s["scale"], s["table"], s["len"])
        if case["op"] == "evict":
            s["to"] = amd.Fp8Cache(s["to_k"], s["to_v"], s["to_scale"], s["to_table"], s["to_len"])
    return s


# ---- one pass --------------------------------------------------------------------------------
def run(state):
    case = state["case"]
    op = case["op"]
    if own:
        amd, cache = state["amd"], state["cache"]
        if op == "append":
            q = amd.append_fp8(cache, state["new_k"], state["new_v"], state["q"], rows=state["rows"], theta=case["theta"])
            return {"q": q, "k": state["k"], "v": state["v"], "scale": state["scale"]}
        if op == "attend":
            out, lse = amd.attend_fp8(cache, state["q"], rows=state["rows"], window=case["window"], sinks=case["sinks"], want_lse=True)
            return {"out": out, "lse": lse}
        if op == "weigh":
            return amd.weigh_fp8(cache, state["q"], state["lse"], state["weight"], rows=state["rows"], window=case["window"],
                                 sinks=case["sinks"])
        kept = amd.evict_fp8(cache, state["weight"], state["to"], case["budget"], case["sinks"], case["recent"],
                             to_weight=state["to_weight"])
        return _evicted(state, kept)
    if op == "append":
        return _plain_append(state, case)
    if op == "attend":
        return _plain_attend(state, case)
    if op == "weigh":
        return _plain_weigh(state, case)
    return _plain_evict(state, case)


def _evicted(s, kept):
    return {"kept": kept, "k": s["to_k"], "v": s["to_v"], "scale": s["to_scale"], "len": s["to_len"], "weight": s["to_weight"]}


def _padded(s):
    """Row index [seqs][most] of every sequence's rows, which of them there are, and the entries they stand for."""
    first, m = s["rows"][:-1, None].long(), (s["rows"][1:] - s["rows"][:-1])[:, None].long()
    j = torch.arange(s["most"], device="cuda")[None]
    return (first + j).clamp_max(s["rows"][-1].long() - 1), j < m, s["len"][:, None] - m + j


def _dense(s, what):
    """Keys or values [seqs][kv][entries][d] in fp32."""
    pool = s[what].view(torch.uint8)[s["table"].clamp_min(0)].view(E4M3).float()
    pool = pool if what == "k" else pool.transpose(3, 4)
    scale = s["scale"][..., 0 if what == "k" else 1][s["table"].clamp_min(0)]
    x = (pool * scale[..., None, None]).transpose(1, 2)
    return x.reshape(x.shape[0], x.shape[1], -1, x.shape[4])


def _visible(s, case, pos, n):
    p = torch.arange(n, device="cuda")
    see = p <= pos[:, :, None]
    if case["window"]:
        see = see & ((p > pos[:, :, None] - case["window"]) | (p < case["sinks"]))
    return see


def _scores(s, case):
    """Scores [seqs][kv][G][most][entries] of the padded rows, and which of them count."""
    index, there, pos = _padded(s)
    heads, kv, d = case["heads"], case["kv"], case["d"]
    k = _dense(s, "k")
    q = s["q"].float()[index].view(index.shape[0], -1, kv, heads // kv, d).permute(0, 2, 3, 1, 4)
    x = torch.matmul(q.reshape(q.shape[0], kv, -1, d), k.transpose(2, 3).contiguous()) / math.sqrt(d)
    see = _visible(s, case, pos, k.shape[2]) & there[:, :, None]
    return x.view(*q.shape[:4], -1), see[:, None, None], index, there


def _plain_attend(s, case):
    x, see, index, there = _scores(s, case)
    x = x.masked_fill_(~see, -math.inf)
    top = x.amax(dim=-1, keepdim=True).clamp_min(-3e38)     # padded rows see nothing
    w = torch.exp(x - top)
    total = w.sum(dim=-1, keepdim=True)
    out = torch.matmul(w.flatten(2, 3), _dense(s, "v")).view(*x.shape[:4], -1) / total
    lse = (top + torch.log(total)).squeeze(-1)
    out = out.permute(0, 3, 1, 2, 4).flatten(2, 3)[there]
    return {"out": out.to(BF16), "lse": lse.permute(0, 3, 1, 2).flatten(2)[there]}


def _plain_weigh(s, case):
    x, see, index, there = _scores(s, case)
    lse = s["lse"][index].view(x.shape[0], x.shape[3], x.shape[1], x.shape[2]).permute(0, 2, 3, 1)
    w = torch.where(see, torch.exp(x - lse[..., None]), 0.0).sum(dim=(2, 3))
    m = s["rows"][1:] - s["rows"][:-1]
    p = torch.arange(w.shape[2], device="cuda")
    before = (p < (s["len"] - m)[:, None])[:, None]
    now = torch.where(before, s["weight"], 0.0) + w
    return s["weight"].copy_(torch.where((p < s["len"][:, None])[:, None], now, s["weight"]))


def _rotate(x, pos, theta):
    """Pairs (i, i + d / 2) of rows [...][heads][d] turned by pos * theta^(-2 i / d); the angle in 64 bits."""
    if not theta:
        return x.float()
    half = x.shape[-1] // 2
    angle = pos[..., None].double() * theta ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
    c, n = torch.cos(angle).float()[..., None, :], torch.sin(angle).float()[..., None, :]
    a, b = x.float().split(half, dim=-1)
    return torch.cat([a * c - b * n, b * c + a * n], dim=-1)


def _plain_append(s, case):
    index, there, pos = _padded(s)
    q = _rotate(s["q"], pos[there], case["theta"]).to(BF16)
    m = (s["rows"][1:] - s["rows"][:-1])[:, None].long()
    length = s["len"][:, None].long()
    first = length - m
    pages = first // PAGE + torch.arange(_pages(s["most"]) + 1, device="cuda")            # [seqs][touched]
    touched = pages * PAGE < length
    ids = s["table"].gather(1, pages.clamp_max(s["table"].shape[1] - 1))[touched].long()
    p = pages[:, :, None] * PAGE + torch.arange(PAGE, device="cuda")
    row = (s["rows"][:-1, None, None].long() + p - first[:, :, None])[touched]
    old = (p < first[:, :, None])[touched]
    new = ~old & (p < length[:, :, None])[touched]
    for what, x in (("k", _rotate(s["new_k"], pos[there], case["theta"])), ("v", s["new_v"].float())):
        x = x[row.clamp(0, x.shape[0] - 1)].transpose(1, 2)                              # [touched][kv][64][d]
        keep, put = old[:, None, :, None], new[:, None, :, None]
        pool, at = s[what].view(torch.uint8), 0 if what == "k" else 1
        was = pool[ids] if what == "k" else pool[ids].transpose(2, 3)
        e_new = _exponent(torch.where(put, x.abs(), 0.0).amax(dim=(2, 3)))
        e_old = torch.frexp(s["scale"][ids, :, at])[1] - 1
        e = torch.where(old[:, :1], torch.maximum(e_old, e_new), e_new)
        moved = was.contiguous().view(E4M3).float() * _power(e_old - e)[:, :, None, None]
        codes = torch.where(keep, moved, x * _power(-e)[:, :, None, None]).clamp(-448, 448).to(E4M3).view(torch.uint8)
        codes = torch.where(keep | put, codes, was)
        pool[ids] = codes if what == "k" else codes.transpose(2, 3)
        s["scale"][ids, :, at] = _power(e)
    return {"q": q, "k": s["k"], "v": s["v"], "scale": s["scale"]}


def _plain_evict(s, case):
    seqs, kv, width = s["weight"].shape
    budget, sinks, recent = case["budget"], case["sinks"], case["recent"]
    p = torch.arange(width, device="cuda")
    length = s["len"][:, None, None]
    rank = torch.where((p < sinks) | (p >= length - recent), math.inf, s["weight"])
    rank = torch.where(p < length, rank, -1.0)
    order = torch.sort(rank, dim=2, descending=True, stable=True)[1][:, :, :budget]        # equal ones: the lowest first
    if order.shape[2] < budget:
        order = torch.cat([order, torch.full((seqs, kv, budget - order.shape[2]), width, device="cuda")], dim=2)
    kept = torch.where(order < length, order, width).sort(dim=2)[0]
    count = s["len"].clamp_max(budget)
    there = kept < width
    slots = s["to_table"].shape[1] * PAGE
    pad = torch.full((seqs, kv, slots - budget), width, device="cuda")
    source = torch.cat([kept, pad], dim=2)
    ids = s["to_table"].reshape(-1).long()
    used = (torch.arange(s["to_table"].shape[1], device="cuda") * PAGE < count[:, None]).reshape(-1)
    live = (source < width).view(seqs, kv, -1, PAGE, 1).transpose(1, 2).reshape(len(ids), kv, PAGE, 1)[used]
    ids = ids[used]
    for what, at in (("k", 0), ("v", 1)):
        x = _dense(s, what).gather(2, source.clamp_max(width - 1)[..., None].expand(-1, -1, -1, case["d"]))
        x = x.view(seqs, kv, -1, PAGE, case["d"]).transpose(1, 2).reshape(-1, kv, PAGE, case["d"])[used]
        codes, e = _token_codes(torch.where(live, x, 0.0))
        pool = s["to_" + what].view(torch.uint8)
        was = pool[ids] if what == "k" else pool[ids].transpose(2, 3)
        codes = torch.where(live, codes, was)
        pool[ids] = codes if what == "k" else codes.transpose(2, 3)
        s["to_scale"][ids, :, at] = _power(e)
    s["to_len"].copy_(count)
    w = s["weight"].gather(2, source.clamp_max(width - 1))
    s["to_weight"].copy_(torch.where(source < width, w, s["to_weight"]))
    return _evicted(s, torch.where(there, kept, -1).to(torch.int32))


# ---- what a pass cannot do without ------------------------------------------------------------
def _seen(m, n, window, sinks):
    """(pairs of a row and an entry that it sees, entries that any row sees) of one sequence."""
    if not window:
        return m * n - m * (m - 1) // 2, n
    pairs = 0
    for pos in range(n - m, n):
        low = max(0, pos - window + 1)
        pairs += pos + 1 - low + min(low, sinks)
    low = max(0, n - m - window + 1)
    return pairs, n - low + min(low, sinks)


def work(case):
    heads, kv, d = case["heads"], case["kv"], case["d"]
    sizes = _sizes(case)
    rows = sum(m for m, _ in sizes)
    if case["op"] == "append":
        return {"bytes": rows * d * (4 * heads + 2 * kv * 3), "flops": rows * d * (3 * heads + 8 * kv)}
    if case["op"] == "evict":
        kept = sum(min(n, case["budget"]) for _, n in sizes)
        return {"bytes": kv * (4 * sum(n for _, n in sizes) + kept * (4 * d + 8)), "flops": kv * (sum(n for _, n in sizes) + 4 * kept * d)}
    seen = [_seen(m, n, case["window"], case["sinks"]) for m, n in sizes]
    pairs, entries = sum(a for a, _ in seen), sum(b for _, b in seen)
    if case["op"] == "weigh":
        return {"bytes": kv * entries * (d + 8) + rows * heads * (2 * d + 4), "flops": heads * pairs * (2 * d + 4)}
    return {"bytes": kv * entries * 2 * d + rows * heads * (4 * d + 4), "flops": heads * pairs * (4 * d + 5)}


# ---- the definitions in 64 bits --------------------------------------------------------------
def _round_e4m3(v):
    """Nearest value with 4 significant bits (fewer below 2^-6), ties to the even one."""
    step = torch.exp2((torch.frexp(v)[1].double() - 1).clamp_min(-6.0) - 3)
    return torch.round(v / step) * step


def _least_scale(top):
    e = LEAST
    if top > 0:
        e = max(LEAST, math.frexp(top)[1] - 9)
        while 448.0 * 2.0 ** e < top:
            e += 1
    return 2.0 ** e


def _entries(s, i, h, what, n):
    """Keys or values [n][d] of one sequence and head in 64 bits."""
    got = []
    for j in range(_pages(n)):
        page = int(s["host_table"][i][j])
        x = s[what][page, h].double() * s["host_scale"][page][h][0 if what == "k" else 1]
        got.append(x if what == "k" else x.t())
    return torch.cat(got)[:n]


def _mask(n, m, window, sinks):
    pos = torch.arange(n - m, n, device="cuda")[:, None]
    p = torch.arange(n, device="cuda")[None]
    far = torch.zeros_like(p > pos) if not window else (pos - p >= window) & (p >= sinks)
    return (p <= pos) & ~far


def _turned(x, pos, theta):
    x = x.double()
    if not theta:
        return x
    half = x.shape[-1] // 2
    z = torch.complex(x[..., :half].contiguous(), x[..., half:].contiguous())
    freq = torch.tensor([theta ** (-2.0 * i / (2 * half)) for i in range(half)], dtype=torch.float64, device="cuda")
    angle = pos.double()[:, None, None] * freq
    z = z * torch.polar(torch.ones_like(angle), angle)
    return torch.cat([z.real, z.imag], dim=-1)


def exact(case, seed):
    sizes, kv, d = _sizes(case), case["kv"], case["d"]
    heads, G = case["heads"], case["heads"] // case["kv"]
    pages = sum(_pages(n) for _, n in sizes) * kv
    if (pages if case["op"] in ("attend", "weigh") else 0) > 50000 or (case["op"] == "evict" and pages > 20000):
        return None                                         # page by page that takes too long
    s = _inputs(case, seed)
    s["host_table"], s["host_scale"] = s["table"].tolist(), s["scale"].double().tolist()
    starts = s["rows"].tolist()
    if case["op"] == "append":
        return _exact_append(s, case, sizes, starts)
    if case["op"] == "evict":
        return _exact_evict(s, case, sizes)
    n_rows = starts[-1]
    out = torch.zeros(n_rows, heads, d, dtype=torch.float64, device="cuda")
    lse = torch.zeros(n_rows, heads, dtype=torch.float64, device="cuda")
    weight = s["weight"].double() if case["op"] == "weigh" else None
    for i, (m, n) in enumerate(sizes):
        see = _mask(n, m, case["window"], case["sinks"])
        a, b = starts[i], starts[i + 1]
        for h in range(kv):
            k = _entries(s, i, h, "k", n).t().contiguous()
            total = torch.zeros(n, dtype=torch.float64, device="cuda")
            for g in range(h * G, (h + 1) * G):
                x = torch.mm(s["q"][a:b, g].double(), k) / math.sqrt(d)
                if case["op"] == "weigh":
                    total += (torch.exp(x - s["lse"][a:b, g].double()[:, None]) * see).sum(dim=0)
                else:
                    x[~see] = -math.inf
                    lse[a:b, g] = torch.logsumexp(x, dim=1)
                    if g == h * G:
                        v = _entries(s, i, h, "v", n).contiguous()
                    out[a:b, g] = torch.mm(torch.exp(x - lse[a:b, g][:, None]), v)
            if case["op"] == "weigh":
                weight[i, h, n - m : n] = 0
                weight[i, h, :n] += total
    return weight if case["op"] == "weigh" else {"out": out, "lse": lse}


def _exact_append(s, case, sizes, starts):
    n_rows = starts[-1]
    pos = torch.cat([torch.arange(n - m, n, device="cuda") for m, n in sizes])
    q, new_k = _turned(s["q"], pos, case["theta"]), _turned(s["new_k"], pos, case["theta"])
    codes = {"k": s["k"].double(), "v": s["v"].double()}
    scale = s["scale"].double()
    for i, (m, n) in enumerate(sizes):
        for page in range((n - m) // PAGE, _pages(n)):
            at, lo, hi = s["host_table"][i][page], max(0, n - m - page * PAGE), min(PAGE, n - page * PAGE)
            r = starts[i] + page * PAGE + lo - (n - m)
            for w, (what, x) in enumerate((("k", new_k[r : r + hi - lo]), ("v", s["new_v"][r : r + hi - lo].double()))):
                tops = x.abs().amax(dim=(0, 2)).tolist()
                for h in range(case["kv"]):
                    was = s["host_scale"][at][h][w]
                    now = max(_least_scale(tops[h]), was if lo else 0.0)
                    into = codes[what][at, h] if what == "k" else codes[what][at, h].t()
                    if lo and now != was:
                        into[:lo] = _round_e4m3(into[:lo] * (was / now))
                    into[lo:hi] = _round_e4m3(x[:, h] / now)
                    scale[at, h, w] = now
    return {"q": q, **codes, "scale": scale}


def _exact_evict(s, case, sizes):
    budget, sinks, recent, kv = case["budget"], case["sinks"], case["recent"], case["kv"]
    k, v, scale = s["to_k"].double(), s["to_v"].double(), s["to_scale"].double()
    weight, kept = s["to_weight"].double(), torch.full((len(sizes), kv, budget), -1, dtype=torch.int32, device="cuda")
    to_table, host = s["to_table"].tolist(), s["weight"].cpu().tolist()
    for i, (_, n) in enumerate(sizes):
        for h in range(kv):
            keep = list(range(n))
            if n > budget:
                middle = sorted(range(sinks, n - recent), key=lambda p: (-host[i][h][p], p))[: budget - sinks - recent]
                keep = sorted(list(range(sinks)) + middle + list(range(n - recent, n)))
            at = torch.tensor(keep, device="cuda")
            kept[i, h, : len(keep)] = at.to(torch.int32)
            weight[i, h, : len(keep)] = s["weight"][i, h, at].double()
            for w, what in enumerate("kv"):
                x = _entries(s, i, h, what, n)[at]
                tops = [float(part.abs().max()) for part in x.split(PAGE)]
                for j, part in enumerate(x.split(PAGE)):
                    page, by = to_table[i][j], _least_scale(tops[j])
                    into = k[page, h] if what == "k" else v[page, h].t()
                    into[: len(part)] = _round_e4m3(part / by)
                    scale[page, h, w] = by
    return {"kept": kept, "k": k, "v": v, "scale": scale, "len": torch.tensor([min(n, budget) for _, n in sizes], dtype=torch.int32),
            "weight": weight}
