"""What a decode or prefill worker does with a paged cache once it holds it: attention of new tokens over the
pages, and the sharing, taking, giving back, compacting and copying of pages.

``run`` is one call sequence of a user's program.  Where ``own`` is false it computes the same in elementary
torch operations, in 32 bits, rounded once at the end.

Sizes follow the caches of ``paper_2607_28633_amd/workloads.py`` (8 KV heads of 128, heads of 64 and 256, an MLA
latent of 576 of which 512 are the value, pages of 16 and 64 tokens), with query heads in groups as such models
have them.  Lengths follow from the case alone, contents and page assignments from the seed of ``prepare``.
"""
import math
import random

import torch

own = False

DTYPE = {"bf16": torch.bfloat16, "fp16": torch.float16, "e4m3": torch.float8_e4m3fn}
SIZE = {"bf16": 2, "fp16": 2, "e4m3": 1}


def _attend(name, kind, **over):
    c = {"name": name, "kind": kind, "type": "bf16", "cache": "bf16", "planes": 2, "kv": 8, "group": 8, "dim": 128,
         "value": 128, "page": 16, "major": "slot", "reqs": 1, "median": 4096, "sigma": 0.0, "low": 1, "high": 1 << 20,
         "lens": 1, "new": 1, "window": 0, "sinks": 0}
    c.update(over)
    return c


def _pages(name, kind, **over):
    c = {"name": name, "kind": kind, "layers": 4, "planes": 2, "kv": 8, "dim": 128, "page": 16, "rows": 16, "beams": 4,
         "median": 1024, "sigma": 0.5, "low": 1, "high": 1 << 17, "lens": 1, "slack": 1.25}
    c.update(over)
    return c


def listed():
    return [
        # The first token after a short chat prompt, an 8B-shaped model: the smallest call, all latency.
        _attend("decode-chat", "decode", group=4, median=100),
        # One layer of a 70B-shaped model's decode step: 8 requests of uneven length.
        _attend("decode-batch8", "decode", reqs=8, sigma=0.6, low=1024, high=8192),
        # One request with a very long context: few rows, so the length itself has to be split.
        _attend("decode-long", "decode", median=131072),
        # A large batch over an 8-bit cache.
        _attend("decode-e4m3", "decode", cache="e4m3", reqs=64, sigma=1.0, low=256, high=16384),
        # Sliding-window layers that keep the first 4 tokens visible, in a head-major pool.
        _attend("decode-window", "decode", dim=64, value=64, reqs=32, sigma=1.0, low=512, high=16384, window=128, sinks=4,
                major="head"),
        # An MLA cache: one latent of 576 a token shared by 16 heads (a share of 8-way tensor parallelism).
        _attend("decode-mla", "decode", planes=1, kv=1, group=16, dim=576, value=512, page=64, reqs=32, sigma=1.0, low=512,
                high=16384),
        # A whole prompt of 8192 tokens at once.
        _attend("prompt-8k", "prompt", median=8192, new=8192),
        # Prompts of uneven length through sliding-window layers with first tokens kept.
        _attend("prompt-window", "prompt", dim=64, value=64, reqs=5, median=3000, sigma=0.5, low=700, high=8192, new=8192,
                window=128, sinks=4),
        # Chunked prefill of a tensor-parallel share: 512 new tokens (fewer where a prompt ends) of each of six
        # requests that already hold a long cache.
        _attend("prompt-chunks", "prompt", type="fp16", cache="fp16", kv=1, reqs=6, median=5000, sigma=0.8, low=300,
                high=16384, new=512),
        # A step of beam search: the old beams give their pages back, every prompt's new ones branch off, each takes
        # a token more, and the partial pages are copied in all layers.
        _pages("pages-beams", "beams", layers=16, rows=16, beams=8, median=1000),
        # Requests leave and others come: bookkeeping alone, over a pool of many pages.
        _pages("pages-turnover", "turnover", layers=0, rows=512, beams=1, median=2000, sigma=1.0),
        # Half of a batch has left, the rest moves together so that the upper part of the pool can be given away.
        _pages("pages-compact", "compact", layers=8, rows=64, beams=1, median=1000, sigma=0.7),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        c = _draw(rng)
        if _fits(c):
            return c


def _draw(rng):
    kind = rng.choice(["decode", "decode", "decode", "prompt", "prompt", "beams", "turnover", "compact"])
    lens = rng.randint(1, 1 << 20)
    if kind in ("decode", "prompt"):
        t, cache = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "e4m3"), ("fp16", "e4m3")])
        dim = rng.choice([64, 96, 128, 128, 128, 256])
        window = rng.choice([0, 0, 0, 128, 1000, 4096])
        c = _attend("", kind, type=t, cache=cache, kv=rng.choice([1, 2, 4, 8, 8]), group=rng.choice([1, 2, 4, 5, 8, 8, 16]),
                    dim=dim, value=dim, page=rng.choice([1, 16, 16, 16, 24, 32, 64, 256]), major=rng.choice(["slot", "slot", "head"]),
                    sigma=rng.choice([0.0, 0.7, 1.0]), high=131072, lens=lens, window=window,
                    sinks=rng.choice([0, 1, 4, 20]) if window else 0)
        if kind == "decode":
            c.update(reqs=_log_int(rng, 1, 256), median=_log_int(rng, 1, 65536))
            if rng.random() < 0.2:
                c.update(planes=1, kv=1, group=rng.choice([8, 16, 32, 64, 128]), dim=576, value=512, page=rng.choice([16, 64]))
        else:
            c.update(reqs=_log_int(rng, 1, 16), median=_log_int(rng, 16, 16384), new=_log_int(rng, 16, 8192))
    else:
        c = _pages("", kind, lens=lens, page=rng.choice([1, 16, 16, 32, 64]), kv=rng.choice([1, 2, 8, 8]),
                   dim=rng.choice([64, 128, 128, 256]), layers=rng.randint(1, 32), rows=_log_int(rng, 1, 256),
                   beams=_log_int(rng, 1, 16), median=_log_int(rng, 16, 8192), sigma=rng.choice([0.0, 0.5, 1.0]),
                   slack=rng.choice([1.1, 1.25, 2.0]))
        if kind == "turnover":
            c.update(layers=0, beams=1, rows=_log_int(rng, 1, 2048))
        elif kind == "compact":
            c.update(beams=1)
    del c["name"]
    return c


def _fits(c):
    """A drawn case costs no more than the largest listed one: in work, and in the plain form's padded scores."""
    w = work(c)
    if w["bytes"] > 1.3e9 or w["flops"] > 1.1e12:
        return False
    if c["kind"] in ("decode", "prompt"):
        lens = _lengths(c)
        most = max(len(_visible(c, n)) for n in lens) if c["kind"] == "decode" else max(lens)
        new = 1 if c["kind"] == "decode" else min(max(lens), c["new"])
        wide = c["reqs"] * most * c["kv"] * (4 * c["dim"] + 3 * new * c["group"])
        return wide <= 1.4e10 and 1.2 * sum(lens) * c["planes"] * c["kv"] * c["dim"] * SIZE[c["cache"]] < 8e9
    pages = c["slack"] * sum(-(-n // c["page"]) for n in _lengths(c)) + 2 * c["rows"] * c["beams"]
    return pages * max(1, c["layers"]) * c["planes"] * c["page"] * c["kv"] * c["dim"] * 2 < 8e9


# ---- what follows from a case alone -----------------------------------------------------------------------

def _lengths(c):
    rng = random.Random(c["lens"])
    n = c["reqs"] if "reqs" in c else c["rows"]
    return [min(c["high"], max(c["low"], int(round(c["median"] * math.exp(c["sigma"] * rng.gauss(0, 1)))))) for _ in range(n)]


def _visible(c, n):
    """Cache positions that the last of n tokens sees."""
    start = max(0, n - c["window"]) if c["window"] else 0
    return [*range(min(c["sinks"], start)), *range(start, n)] if c["window"] else range(n)


def _seen(c, n, new):
    """How many (row, key) pairs `new` last tokens of n make, and how many keys any of them sees."""
    pairs = 0
    if not c["window"]:
        pairs = new * n - new * (new - 1) // 2
        return pairs, n
    w, s = c["window"], c["sinks"]
    for p in range(n - new, n):
        start = max(0, p + 1 - w)
        pairs += p + 1 - start + min(s, start)
    start = max(0, n - new + 1 - w)
    return pairs, n - start + min(s, start)


def _moved(c):
    """Pages that a pass over page bookkeeping copies, and table entries that it reads or writes."""
    lens, p = _lengths(c), c["page"]
    entries = sum(-(-n // p) for n in lens)
    if c["kind"] == "beams":
        return c["beams"] * sum(1 for n in lens if n % p), 3 * c["beams"] * entries
    if c["kind"] == "turnover":
        return 0, 3 * entries
    return None, 2 * sum(-(-n // p) for n in lens[::2])


def work(case):
    c = case
    if c["kind"] in ("decode", "prompt"):
        heads, out = c["kv"] * c["group"], c["value"]
        width = c["dim"] if c["planes"] == 1 else c["dim"] + c["value"]
        rows = pairs = keys = 0
        for n in _lengths(c):
            new = 1 if c["kind"] == "decode" else min(n, c["new"])
            a, b = _seen(c, n, new)
            rows, pairs, keys = rows + new, pairs + a, keys + b
        return {"bytes": keys * c["kv"] * width * SIZE[c["cache"]] + rows * heads * ((c["dim"] + out) * 2 + 4)
                + 4 * -(-keys // c["page"]) + 8 * c["reqs"],
                "flops": 2 * heads * (c["dim"] + out) * pairs}
    block = c["planes"] * c["page"] * c["kv"] * c["dim"] * 2
    moved, entries = _moved(c)
    pages = int(c["slack"] * sum(-(-n // c["page"]) for n in _lengths(c))) + 2 * c["rows"] * c["beams"]
    if moved is None:                                                  # the rest lies over the whole pool
        live = entries // 2
        moved = live * (pages - live) // pages
    return {"bytes": 2 * c["layers"] * moved * block + 4 * entries + 4 * pages, "flops": 0}


# ---- what a user's program has in hand ----------------------------------------------------------------------

def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 6151 + 29)
    return _attention_state(case, gen) if case["kind"] in ("decode", "prompt") else _page_state(case, gen)


def _normal(shape, name, gen):
    t = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float16 if name == "e4m3" else DTYPE[name])
    return t.to(DTYPE[name]) if name == "e4m3" else t


def _hand_out(need, pages, gen):
    """Every row takes the next pages of a random permutation; unused entries are -1."""
    perm = torch.randperm(pages, generator=gen, device="cuda", dtype=torch.int32)
    bt = torch.full((len(need), max([1] + need)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for r, k in enumerate(need):
        bt[r, :k] = perm[at:at + k]
        at += k
    return bt


def _attention_state(c, gen):
    lens = _lengths(c)
    need = [-(-n // c["page"]) for n in lens]
    pages = math.ceil(1.1 * sum(need))
    new = [1 if c["kind"] == "decode" else min(n, c["new"]) for n in lens]
    heads, total = c["kv"] * c["group"], sum(new)
    slot = (c["kv"], c["page"]) if c["major"] == "head" else (c["page"], c["kv"])
    s = {"case": c, "lens": torch.tensor(lens, dtype=torch.int32, device="cuda"), "tables": _hand_out(need, pages, gen),
         "pool": _normal((1, pages, c["planes"]) + slot + (c["dim"],), c["cache"], gen),
         "starts": torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32, device="cuda"),
         "new": new, "total": total}
    # queries as the projection leaves them: in front of the keys and values of the same tokens (MLA: on their own)
    width = heads * c["dim"] + (2 * c["kv"] * c["dim"] if c["planes"] == 2 else 0)
    s["qkv"] = _normal((total, width), c["type"], gen) * 1.5
    s["q"] = s["qkv"][:, :heads * c["dim"]].view(total, heads, c["dim"])
    s["out"] = torch.empty((total, heads, c["value"]), dtype=DTYPE[c["type"]], device="cuda")
    s["lse"] = torch.empty((total, heads), dtype=torch.float32, device="cuda")
    s["scale"] = 1.0 / math.sqrt(c["dim"] if c["planes"] == 2 else 192)
    s["k_scale"], s["v_scale"] = (0.75, 1.25) if c["cache"] == "e4m3" else (1.0, 1.0)
    return s


def _page_state(c, gen):
    lens = _lengths(c)
    p, rows, beams = c["page"], c["rows"], c["beams"]
    need = [-(-n // p) for n in lens]
    pages = int(c["slack"] * sum(need)) + 2 * rows * beams
    own_pages = _hand_out(need, pages, gen)
    total = rows * (1 + beams) if c["kind"] == "beams" else rows
    tables = torch.full((total, own_pages.shape[1] + 1), -1, dtype=torch.int32, device="cuda")
    tables[:rows, :own_pages.shape[1]] = own_pages
    seq = torch.zeros(total, dtype=torch.int32, device="cuda")
    seq[:rows] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    if c["kind"] == "compact":                                         # every second request has left
        tables[1::2] = -1
        seq[1::2] = 0
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    named = tables[tables >= 0].long()
    refs.scatter_add_(0, named, torch.ones_like(named, dtype=torch.int32))
    s = {"case": c, "tables": tables, "lens": seq, "refs": refs,
         "pairs": torch.zeros((max(pages // 2 + 1, total), 2), dtype=torch.int32, device="cuda")}
    if c["layers"]:
        s["pool"] = torch.empty((c["layers"], pages, c["planes"], p, c["kv"], c["dim"]), dtype=torch.int16, device="cuda")
        s["pool"].random_(-32768, 32768, generator=gen)
    if c["kind"] == "beams":
        s["parents"] = torch.randint(0, rows, (rows * beams,), generator=gen, device="cuda", dtype=torch.int32)
        s["children"] = torch.arange(rows, total, device="cuda", dtype=torch.int32)
    elif c["kind"] == "turnover":
        leave = torch.randperm(rows, generator=gen, device="cuda", dtype=torch.int32)[:max(1, rows // 3)]
        s["leave"] = leave.contiguous()
        s["come"] = s["lens"][leave.long()].flip(0).contiguous()
    return s


# ---- one pass -------------------------------------------------------------------------------------------------

def run(state):
    kind = state["case"]["kind"]
    if own:
        return _own_attention(state) if kind in ("decode", "prompt") else _OWN[kind](state)
    return _plain_attention(state) if kind in ("decode", "prompt") else _PLAIN[kind](state)


def _own_attention(s):
    c = s["case"]
    if "call" not in s:                                                # the handle that a serving loop keeps
        from paper_2607_28633_amd import topkv
        cache = topkv.pool_view(s["pool"], 0, s["tables"], s["tables"].shape[1], 0, c["major"] == "head")
        options = topkv.attention_options(s["q"], s["out"], kv_dtype=DTYPE[c["cache"]], kv_heads=c["kv"], scale=s["scale"],
                                          window=c["window"], sinks=c["sinks"], k_scale=s["k_scale"], v_scale=s["v_scale"])
        room = topkv.topkv_attention_workspace_bytes(cache, options, c["reqs"], s["total"])
        s["work"] = torch.empty(room, dtype=torch.uint8, device="cuda")
        if c["kind"] == "decode":
            s["call"] = topkv.prepare_attention_decode(cache, options, c["reqs"], s["lens"], s["q"], s["out"], s["work"],
                                                       lse=s["lse"])
        else:
            s["call"] = topkv.prepare_attention_prompt(cache, options, c["reqs"], s["lens"], s["starts"], s["total"], s["q"],
                                                       s["out"], s["work"], lse=s["lse"])
    s["call"]()
    return {"out": s["out"], "lse": s["lse"]}


def _own_handles(s):
    from paper_2607_28633_amd import topkv
    if "owner" not in s:
        c = s["case"]
        s["owner"] = topkv.page_owner(s["refs"], s["tables"], s["lens"], page_size=c["page"])
        s["work"] = torch.empty(topkv.topkv_pages_workspace_bytes(s["owner"]), dtype=torch.uint8, device="cuda")
        s["result"] = torch.zeros(4, dtype=torch.int32, device="cuda")
    return topkv


def _own_beams(s):
    topkv = _own_handles(s)
    c, kids = s["case"], s["children"]
    n = kids.shape[0]
    topkv.topkv_pages_free(s["owner"], n, kids, s["result"])
    topkv.topkv_pages_fork(s["owner"], n, s["parents"], kids, s["pairs"], s["work"], s["result"])
    topkv.topkv_copy_pages(s["pool"], s["pool"], 0, c["layers"], s["pairs"], n, s["result"][1:])
    longer = s["lens"][c["rows"]:] + 1                                 # the children's rows come last
    topkv.topkv_pages_grow(s["owner"], n, kids, longer, s["pairs"], s["work"], s["result"])
    return {"tables": s["tables"], "lens": s["lens"], "refs": s["refs"], "pool": s["pool"]}


def _own_turnover(s):
    topkv = _own_handles(s)
    n = s["leave"].shape[0]
    topkv.topkv_pages_free(s["owner"], n, s["leave"], s["result"])
    topkv.topkv_pages_grow(s["owner"], n, s["leave"], s["come"], s["pairs"], s["work"], s["result"])
    return {"tables": s["tables"], "lens": s["lens"], "refs": s["refs"]}


def _own_compact(s):
    """The batch as it is stays for the next pass: what is compacted are copies of the tables and counts."""
    from paper_2607_28633_amd import topkv
    c = s["case"]
    tables, refs = s["tables"].clone(), s["refs"].clone()
    owner = topkv.page_owner(refs, tables, s["lens"], page_size=c["page"])
    if "work" not in s:
        s["work"] = torch.empty(topkv.topkv_pages_workspace_bytes(owner), dtype=torch.uint8, device="cuda")
        s["result"] = torch.zeros(4, dtype=torch.int32, device="cuda")
    topkv.topkv_pages_compact(owner, s["pairs"], s["work"], s["result"])
    topkv.topkv_copy_pages(s["pool"], s["pool"], 0, c["layers"], s["pairs"], s["pairs"].shape[0], s["result"][1:])
    return {"tables": tables, "refs": refs, "pool": s["pool"]}


_OWN = {"beams": _own_beams, "turnover": _own_turnover, "compact": _own_compact}


# ---- the same in elementary torch operations -------------------------------------------------------------------

def _plain_attention(s):
    """All requests at once, padded to the longest."""
    c = s["case"]
    lens = s["lens"].long()
    new = torch.diff(s["starts"]).long()
    most = 1 if c["kind"] == "decode" else max(s["new"])
    p = c["page"]
    # keys: of one new token only the visible ones are gathered, of several all
    if c["kind"] == "decode" and c["window"]:
        start = (lens - c["window"]).clamp(min=0)
        first = start.clamp(max=c["sinks"])
        i = torch.arange(min(s["tables"].shape[1] * p, c["window"] + c["sinks"]), device="cuda")
        at = torch.where(i < first[:, None], i, start[:, None] - first[:, None] + i)
    else:
        at = torch.arange(s["tables"].shape[1] * p, device="cuda").expand(len(lens), -1)
    there = at < lens[:, None]
    page = s["tables"].long().gather(1, (at // p).clamp(max=s["tables"].shape[1] - 1)).clamp(min=0)
    pool, slot = s["pool"][0], at % p
    pool = pool.transpose(2, 3) if c["major"] == "head" else pool
    if c["cache"] == "e4m3":
        pool = pool.view(torch.uint8)
    k = pool[page, 0, slot]                                            # [request, key, head, dim]
    v = pool[page, 1, slot] if c["planes"] == 2 else k[..., :c["value"]]
    if c["cache"] == "e4m3":
        k, v = k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn)
    k, v = k.float() * s["k_scale"], v.float() * s["v_scale"]
    # queries, padded to the most new tokens of any request
    t = torch.arange(most, device="cuda")
    row = (s["starts"][:-1, None].long() + t).clamp(max=s["total"] - 1)
    q = s["q"].float()[row].view(len(lens), most, c["kv"], c["group"], c["dim"]).permute(0, 2, 3, 1, 4)
    q = q.reshape(len(lens), c["kv"], c["group"] * most, c["dim"])
    score = torch.matmul(q, k.permute(0, 2, 3, 1)).mul_(s["scale"]).view(len(lens), c["kv"], c["group"], most, -1)
    pos = lens[:, None] - new[:, None] + t                             # [request, new token]
    keep = there[:, None, :] & (at[:, None, :] <= pos[:, :, None])
    if c["window"]:
        keep &= (at[:, None, :] > pos[:, :, None] - c["window"]) | (at[:, None, :] < c["sinks"])
    score.masked_fill_(~keep[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    score.sub_(top).exp_()
    total = score.sum(-1, keepdim=True)
    got = torch.matmul(score.view(len(lens), c["kv"], c["group"] * most, -1), v.permute(0, 2, 1, 3))
    got = got.view(len(lens), c["kv"], c["group"], most, c["value"]) / torch.where(total == 0, 1.0, total)
    lse = (top + total.log()).squeeze(-1)
    real = (t < new[:, None])
    out = got.permute(0, 3, 1, 2, 4).reshape(len(lens), most, c["kv"] * c["group"], c["value"])[real]
    return {"out": out.to(DTYPE[c["type"]]), "lse": lse.permute(0, 3, 1, 2).reshape(len(lens), most, -1)[real]}


def _count(lens, page):
    return (lens + (page - 1)) // page


def _plain_free(s, rows):
    rows, i = rows.long(), torch.arange(s["tables"].shape[1], device="cuda")
    held = s["tables"][rows]
    used = i < _count(s["lens"][rows], s["case"]["page"])[:, None]
    s["refs"].scatter_add_(0, held.clamp(min=0).long().view(-1), -used.int().view(-1))
    s["tables"][rows] = torch.where(used, -1, held)
    s["lens"][rows] = 0


def _plain_take(s, rows, have, want, entries):
    """The lowest free pages, in order, into entries [have, want) of the rows."""
    i = torch.arange(entries.shape[1], device="cuda")
    gap = (i >= have[:, None]) & (i < want[:, None])
    free = (s["refs"] == 0).nonzero().view(-1).int()
    rank = gap.view(-1).cumsum(0).view(gap.shape) - 1
    taken = free[rank.clamp(min=0)]
    s["refs"].scatter_add_(0, taken.view(-1).long(), gap.int().view(-1))
    s["tables"][rows] = torch.where(gap, taken, entries)


def _plain_beams(s):
    c, kids, parents = s["case"], s["children"].long(), s["parents"].long()
    p = c["page"]
    _plain_free(s, kids)
    n, held = s["lens"][parents], s["tables"][parents]
    whole = n // p
    i = torch.arange(held.shape[1], device="cuda")
    shared = i < whole[:, None]
    s["refs"].scatter_add_(0, held.clamp(min=0).long().view(-1), shared.int().view(-1))
    _plain_take(s, kids, whole, _count(n, p), torch.where(shared, held, -1))
    s["lens"][kids] = n
    part = (n % p != 0).nonzero().view(-1)
    src, dst = held[part, whole[part].long()].long(), s["tables"][kids[part], whole[part].long()].long()
    s["pool"][:, dst] = s["pool"][:, src]
    _plain_take(s, kids, _count(n, p), _count(n + 1, p), s["tables"][kids])
    s["lens"][kids] = n + 1
    return {"tables": s["tables"], "lens": s["lens"], "refs": s["refs"], "pool": s["pool"]}


def _plain_turnover(s):
    rows, p = s["leave"].long(), s["case"]["page"]
    _plain_free(s, rows)
    _plain_take(s, rows, torch.zeros_like(s["come"]), _count(s["come"], p), s["tables"][rows])
    s["lens"][rows] = s["come"]
    return {"tables": s["tables"], "lens": s["lens"], "refs": s["refs"]}


def _plain_compact(s):
    live = s["refs"] > 0
    count = int(live.sum())
    low = (~live[:count]).nonzero().view(-1)
    high = (live[count:].nonzero().view(-1) + count).flip(0)           # the highest page goes to the lowest free one
    to = torch.arange(live.shape[0], device="cuda", dtype=torch.int32)
    to[high] = low.int()
    refs, tables = s["refs"].clone(), s["tables"].clone()
    refs[low] = refs[high]
    refs[high] = 0
    tables = torch.where(tables >= 0, to[tables.clamp(min=0).long()], tables)
    s["pool"][:, low] = s["pool"][:, high]
    return {"tables": tables, "refs": refs, "pool": s["pool"]}


_PLAIN = {"beams": _plain_beams, "turnover": _plain_turnover, "compact": _plain_compact}


# ---- the definition in 64 bits ---------------------------------------------------------------------------------

def exact(case, seed):
    """Attention one request and KV head at a time; page bookkeeping is whole numbers and moved words."""
    c = case
    if c["kind"] not in ("decode", "prompt"):
        return None
    s = prepare(case, seed)
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    row = 0
    for r, n in enumerate(_lengths(c)):
        new = s["new"][r]
        block = s["pool"][0][s["tables"][r, :-(-n // c["page"])].long()] if c["cache"] != "e4m3" else \
            s["pool"][0].view(torch.uint8)[s["tables"][r, :-(-n // c["page"])].long()].view(torch.float8_e4m3fn)
        for h in range(c["kv"]):
            one = block[:, :, h] if c["major"] == "head" else block[:, :, :, h]
            one = one.double().permute(1, 0, 2, 3).reshape(c["planes"], -1, c["dim"])[:, :n]
            keys = one[0] * s["k_scale"]
            values = one[1] * s["v_scale"] if c["planes"] == 2 else one[0][:, :c["value"]] * s["v_scale"]
            for g in range(c["group"]):
                head = h * c["group"] + g
                for at in range(0, new, 2048):
                    upto = min(new, at + 2048)
                    pos = torch.arange(n - new + at, n - new + upto, device="cuda")[:, None]
                    j = torch.arange(n, device="cuda")[None]
                    sees = j <= pos
                    if c["window"]:
                        sees &= (j > pos - c["window"]) | (j < c["sinks"])
                    x = (s["q"][row + at:row + upto, head].double() @ keys.t()) * s["scale"]
                    x = torch.where(sees, x, -math.inf)
                    lse[row + at:row + upto, head] = torch.logsumexp(x, 1)
                    out[row + at:row + upto, head] = torch.softmax(x, 1) @ values
        row += new
    return {"out": out, "lse": lse}
