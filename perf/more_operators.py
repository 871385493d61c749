"""Workloads of long contexts in the paged key/value cache, as a user of the library runs them.

What a sequence holds in the cache grows with every token, and attention over it reads all of it.  Two ways to read or hold less:
  bounds    of each page that new tokens lie in, the largest and the smallest value of every dim of its keys;
  score     from these, for each new token and page, the largest that the product of a query head and a key of the page can be;
  select    the pages that a new token reads: the first, the last, and those of the highest scores;
  attend    attention of the new tokens over the pages of their lists;
  weigh     adds up how much attention each token gets from the new ones (older calls' share fades);
  evict     keeps, of every sequence, layer and head, the first tokens, the last, and those of the largest weights, and moves them
            together, to pages of their own or to the front of the ones they are in.
A decoder's layer calls append, bounds, score, select, attend for new tokens, or append, attend, weigh; evict is called once in a while,
when a prompt has been read or a pool is full.

Layouts are those of the cache: keys [layer][page][head][token][dim], values [layer][page][head][dim][token], 8-bit caches with a scale for
each token and head; bounds [layer][page][head][2][dim], weights [layer][page][head][token].  Head counts and sizes are those of
perf/operators.py.

Fields: seqs, new (most new tokens of a sequence), past (most tokens before them), ragged (both spread over a quarter of the range and up, one
sequence in seven without a new token), qh, kvh, dim, page (tokens), cache ("bf16" | "s8"), window (0: none), lists (pages of a list), first, last
(pages always read, or tokens always kept); evict: rows, layers, len, keep, inplace.
"""
import math

import torch

own = False     # whether run() makes the framework's calls; otherwise it computes the plain form

DECAY = 0.9
HEADS = ((4, 4, 64), (12, 12, 64), (16, 16, 64), (12, 4, 64), (16, 2, 64), (32, 8, 128), (16, 16, 128), (8, 1, 128), (10, 5, 80))


def _case(name, kind, seqs, new, past, ragged, qh, kvh, dim, page, cache="bf16", window=0, **more):
    return {"name": name, "kind": kind, "seqs": seqs, "new": new, "past": past, "ragged": ragged, "qh": qh, "kvh": kvh, "dim": dim, "page": page,
            "cache": cache, "window": window, **more}


def _evict(name, rows, len, ragged, keep, first, last, layers, kvh, dim, page, cache="bf16", inplace=False):
    return {"name": name, "kind": "evict", "rows": rows, "len": len, "ragged": ragged, "keep": keep, "first": first, "last": last, "layers": layers,
            "kvh": kvh, "dim": dim, "page": page, "cache": cache, "inplace": inplace}


def listed():
    return [
        # a serving batch's next tokens: each one's page is summed up again; latency
        _case("bounds_64x1_h8", "bounds", 64, 1, 8191, True, 8, 8, 128, 64),
        # long documents just read into an 8-bit cache: all their pages
        _case("bounds_documents_4x16385_s8", "bounds", 4, 16385, 100, False, 8, 8, 128, 64, cache="s8"),
        # one conversation's next token, small pages: latency
        _case("score_1x1_h16", "score", 1, 1, 7760, False, 16, 16, 64, 16),
        # a chunk of new tokens behind a long past, shared key/value heads
        _case("score_chunk_500_past_15k_h32", "score", 1, 500, 15000, False, 32, 8, 128, 16),
        # a serving batch's next tokens: a list for each of 8 heads
        _case("select_64x1_h8", "select", 64, 1, 8191, True, 8, 8, 128, 64, lists=32, first=1, last=2),
        # a chunk of new tokens, a list for each of them and each head, of many small pages
        _case("select_chunk_2000_h8", "select", 1, 2000, 13521, False, 8, 8, 128, 16, lists=64, first=1, last=4),
        # a serving batch's next tokens read 2048 of up to 8192 tokens
        _case("attend_64x1_32_pages_h32", "attend", 64, 1, 8191, True, 32, 8, 128, 64, lists=32, first=1, last=2),
        # a chunk of new tokens, each over pages of its own, 8-bit cache
        _case("attend_chunk_257_16_pages_s8", "attend", 1, 257, 15000, False, 32, 8, 128, 64, cache="s8", lists=16, first=1, last=1),
        # a serving batch's next tokens, contexts of all lengths
        _case("weigh_64x1_h32", "weigh", 64, 1, 8191, True, 32, 8, 128, 64),
        # two prompts just read: their last 32 tokens say what counts
        _case("weigh_last_32_of_16k_h32", "weigh", 2, 32, 16000, False, 32, 8, 128, 64),
        # four conversations of a small decoder, to a quarter
        _evict("evict_4x1000_h12", 4, 1000, False, 250, 4, 64, 12, 12, 64, 16),
        # a batch's long contexts in an 8-bit cache
        _evict("evict_8x12k_s8", 8, 12000, True, 2048, 16, 256, 8, 8, 128, 64, cache="s8"),
    ]


def draw(rng):
    def size(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    most = {}       # a drawn case costs at most what the largest listed one of its kind does
    for c in listed():
        most[c["kind"]] = max(most.get(c["kind"], 0), _cost(c))
    while True:
        kind = rng.choice(("bounds", "score", "select", "attend", "weigh", "evict"))
        qh, kvh, dim = rng.choice(HEADS)
        page, cache, ragged = rng.choice((16, 32, 64, 128)), rng.choice(("bf16", "bf16", "s8")), rng.random() < 0.5
        few = rng.random() < 0.5
        new, past = size(1, 4) if few else size(5, 1024), size(1, 100000) if few else rng.choice((0, size(1, 20000)))
        window = rng.choice((0, 0, 0, size(17, 8192))) if kind != "bounds" else 0
        more = {}
        if kind in ("select", "attend"):
            lists = size(2, 128)
            first = rng.randrange(0, min(4, lists))
            more = {"lists": lists, "first": first, "last": rng.randrange(0, min(4, lists - first) + 1)}
        if kind == "evict":
            n = size(30, 16000)
            first = rng.randrange(0, 17)
            c = _evict("", size(1, 32), n, ragged, size(max(8, n // 16), n), first, size(1, 256), rng.choice((1, 4, 12)), kvh, dim, page, cache, rng.random() < 0.3)
        else:
            c = _case("", kind, size(1, 64), new, past, ragged, qh, kvh, dim, page, cache, window, **more)
        del c["name"]
        if _cost(c) <= most[kind] and _pool_bytes(c) <= 3 << 30 and _plain_bytes(c) <= 12 << 30:
            return c


# ---- what a case is made of: the same for every seed --------------------------------------------------------------------------

def _spread(n, at, step):
    return max(1, int(n * (1 - 0.75 * ((at * step) % 1))))


def _lengths(c):
    """(new, past) tokens of each sequence."""
    if not c["ragged"]:
        return [c["new"]] * c["seqs"], [c["past"]] * c["seqs"]
    return ([0 if b % 7 == 5 else _spread(c["new"], b, 0.618034) for b in range(c["seqs"])],
            [_spread(c["past"], b, 0.754878) if c["past"] else 0 for b in range(c["seqs"])])


def _held(c):
    """Tokens of each row of an eviction, and how many of them stay."""
    lens = [_spread(c["len"], b, 0.754878) if c["ragged"] else c["len"] for b in range(c["rows"])]
    return lens, [min(n, c["keep"]) for n in lens]


def _each(c):
    """Bytes of a token's head: its key, and its scale."""
    return c["dim"] * 2 if c["cache"] == "bf16" else c["dim"] + 4


def _seen(c, at):
    """First and last page that a token at this position sees."""
    return (max(0, at + 1 - c["window"]) // c["page"] if c["window"] else 0), at // c["page"]


def _pages(n, page):
    return -(-n // page)


def work(case):
    c = case
    if c["kind"] == "evict":
        lens, kept = _held(c)
        heads = c["layers"] * c["kvh"]
        return {"bytes": heads * (4 * sum(lens) + sum(kept) * (4 * _each(c) + 8 + 4)), "flops": 0}
    new, past = _lengths(c)
    t, h, d = sum(new), c["kvh"], c["dim"]
    some = [(n, p) for n, p in zip(new, past) if n]
    if c["kind"] == "bounds":
        touched = [n + p - p // c["page"] * c["page"] for n, p in some]
        return {"bytes": h * (sum(touched) * _each(c) + sum(_pages(n, c["page"]) for n in touched) * 4 * d), "flops": 0}
    spans = [[_seen(c, p + i) for i in range(n)] for n, p in some]
    pairs = sum(hi - lo + 1 for s in spans for lo, hi in s)     # of a token and a page
    width = max([_pages(n + p, c["page"]) for n, p in zip(new, past)] + [1])
    q = t * c["qh"] * d * 2
    if c["kind"] == "score":
        pages = sum(s[-1][1] - s[0][0] + 1 for s in spans)
        return {"bytes": pages * h * 4 * d + q + t * h * width * 4, "flops": 4 * d * c["qh"] * pairs}
    if c["kind"] == "select":
        return {"bytes": h * 4 * (pairs + t * c["lists"]), "flops": 0}
    if c["kind"] == "attend":
        read = [[min(c["lists"], hi - lo + 1) for lo, hi in s] for s in spans]
        distinct = sum(min(sum(r), s[-1][1] - s[0][0] + 1) for r, s in zip(read, spans)) * c["page"]
        return {"bytes": 2 * h * distinct * _each(c) + 2 * q, "flops": 4 * d * c["qh"] * c["page"] * sum(sum(r) for r in read)}
    lens = sum(n + p for n, p in some)
    see = sum(min(p + i + 1, c["window"]) if c["window"] else p + i + 1 for n, p in some for i in range(n))
    keys = sum(min(n + p, n + c["window"] - 1) if c["window"] else n + p for n, p in some)
    return {"bytes": h * (keys * _each(c) + 8 * lens) + q, "flops": 2 * d * c["qh"] * see}


def _cost(c):
    w = work(c)
    return w["flops"] + 60 * w["bytes"] if c["kind"] in ("score", "attend", "weigh") else w["bytes"]


def _pool_bytes(c):
    """Keys and values of all pages."""
    if c["kind"] == "evict":
        lens, kept = _held(c)
        tokens = (sum(lens) + sum(kept) + 2 * c["rows"] * c["page"]) * c["layers"]
    else:
        new, past = _lengths(c)
        tokens = sum(new) + sum(past) + c["seqs"] * c["page"]
    return 2 * tokens * c["kvh"] * _each(c)


def _plain_bytes(c):
    """Memory that the plain form takes at its largest, about."""
    if c["kind"] == "evict":
        return 6 * _pool_bytes(c)
    most = c["new"] + c["past"]
    if c["kind"] == "score":
        return c["seqs"] * _pages(most, c["page"]) * (12 * c["new"] * c["qh"] + 8 * c["kvh"] * c["dim"])
    if c["kind"] == "select":
        return 24 * c["seqs"] * c["new"] * c["kvh"] * _pages(most, c["page"])
    if c["kind"] == "attend":
        return c["seqs"] * c["new"] * c["kvh"] * c["lists"] * c["page"] * (16 * c["dim"] + 12 * c["qh"] // c["kvh"])
    if c["kind"] == "weigh":
        return c["seqs"] * most * (8 * c["qh"] * c["new"] + 16 * c["kvh"] * c["dim"])
    return 8 * c["seqs"] * (c["new"] + c["page"]) * c["kvh"] * c["dim"]


# ---- inputs -------------------------------------------------------------------------------------------------------------------

def _pool(c, layers, pages, g):
    """A cache's pages: keys, values (where they are read), and their scales where they are held in 8 bits; bounds and weights."""
    shape = (layers, pages, c["kvh"])
    k_shape, v_shape = (*shape, c["page"], c["dim"]), (*shape, c["dim"], c["page"])
    keys, values = c["kind"] not in ("score", "select"), c["kind"] in ("attend", "evict")
    s = {"k_scale": None, "v_scale": None, "bounds": None, "weight": None}
    for name, size, read in (("k", k_shape, keys), ("v", v_shape, values)):
        if c["cache"] == "s8":
            s[name] = torch.randint(-127, 128, size, generator=g, device="cuda", dtype=torch.int8) if read else torch.zeros(size, device="cuda", dtype=torch.int8)
            s[name + "_scale"] = torch.rand((*shape, c["page"]), generator=g, device="cuda") * 0.012 + 0.01
        else:
            s[name] = torch.randn(size, generator=g, device="cuda", dtype=torch.bfloat16) if read else torch.zeros(size, device="cuda", dtype=torch.bfloat16)
    if c["kind"] in ("bounds", "score"):
        x = torch.randn((*shape, 2, c["dim"]), generator=g, device="cuda") * 0.5
        s["bounds"] = (x + torch.tensor([[2.0], [-2.0]], device="cuda")).to(torch.bfloat16)
    if c["kind"] in ("weigh", "evict"):
        s["weight"] = torch.exp(torch.randn((*shape, c["page"]), generator=g, device="cuda") * 2 - 6)
    return s


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _tables(held, pages, g, width=None):
    """Rows of that many pages each, out of `pages` in any order; several tables of different pages for several lists of `held`."""
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32).cpu()
    width, at, tables = width or max(max(max(h) for h in held), 1), 0, []
    for rows in held:
        table = torch.full((len(rows), width), -1, dtype=torch.int32)
        for b, n in enumerate(rows):
            table[b, :n] = order[at : at + n]
            at += n
        tables.append(table.cuda())
    return tables


def prepare(case, seed):
    c, g = case, torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": c}
    if c["kind"] == "evict":
        lens, kept = _held(c)
        held = [[_pages(n, c["page"]) for n in lens], [0 if c["inplace"] else _pages(n, c["page"]) for n in kept]]
        pages = sum(held[0]) + sum(held[1]) + 2
        s |= _pool(c, c["layers"], pages, g)
        table, to = _tables(held, pages, g)
        return s | {"table": table, "to": table if c["inplace"] else to, "kv_len": _ints(lens), "keep": _ints([c["keep"]] * c["rows"])}
    new, past = _lengths(c)
    held = [_pages(n + p, c["page"]) for n, p in zip(new, past)]
    pages, start = sum(held) + 2, [0]
    s |= _pool(c, 1, pages, g)
    for n in new:
        start.append(start[-1] + n)
    t = start[-1]
    s |= {"table": _tables([held], pages, g)[0], "q_start": _ints(start), "kv_len": _ints([n + p for n, p in zip(new, past)]), "tokens": t}
    if c["kind"] in ("score", "attend", "weigh"):
        s["q"] = (torch.randn((t, c["qh"], c["dim"]), generator=g, device="cuda") * 1.5).to(torch.bfloat16)
    if c["kind"] in ("select", "attend"):
        lo, hi = _spans(s)
        page = torch.arange(s["table"].shape[1], device="cuda")
        hidden = ((page < lo[:, None]) | (page > hi[:, None]))[:, None]
        scores = torch.randn((t, c["kvh"], page.numel()), generator=g, device="cuda").mul_(8).add_(30).masked_fill_(hidden, -math.inf)
        if c["kind"] == "select":
            s["scores"] = scores
        else:
            s["lists"] = _chosen(c, scores, lo, hi)
    return s


def _where(s):
    """Of each new token: its sequence and its place in it."""
    t = torch.arange(s["tokens"], device="cuda")
    start = s["q_start"].long()
    seq = torch.searchsorted(start[1:], t, right=True)
    return seq, s["kv_len"].long()[seq] - start[seq + 1] + t


def _spans(s):
    """Of each new token: the first and the last page that it sees."""
    c, (_, at) = s["case"], _where(s)
    first = (at + 1 - c["window"]).clamp(min=0) // c["page"] if c["window"] else torch.zeros_like(at)
    return first, at // c["page"]


def _chosen(c, scores, lo, hi):
    """The pages of each new token and head: those that are always taken first, then by their score, the lower page first."""
    page = torch.arange(scores.shape[2], device="cuda")
    always = (page < lo[:, None] + c["first"]) | (page > hi[:, None] - c["last"])
    hidden = (page < lo[:, None]) | (page > hi[:, None])
    x = scores.masked_fill((always & ~hidden)[:, None], math.inf).masked_fill_(hidden[:, None], -math.inf)
    n = min(c["lists"], page.numel())
    best = torch.sort(x, dim=-1, descending=True, stable=True).indices[..., :n]
    there = torch.arange(n, device="cuda") < (hi - lo + 1)[:, None, None]
    best = torch.where(there, best, page.numel()).sort(-1).values
    lists = torch.full((*scores.shape[:2], c["lists"]), -1, dtype=torch.int32, device="cuda")
    lists[..., :n] = torch.where(best < page.numel(), best, -1)
    return lists


# ---- one pass -----------------------------------------------------------------------------------------------------------------

def run(state):
    return (_own if own else _plain)[state["case"]["kind"]](state)


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _described(s):
    import paper_2306_16601_amd as sp
    cache = sp.make_cache(s["k"], s["v"], s["k_scale"], s["v_scale"], s["bounds"], s["weight"])
    return sp, cache, None if "q_start" not in s else sp.make_batch(s["q_start"], s["kv_len"], s["table"])


def _own_bounds(s):
    sp, cache, batch = _described(s)
    sp.spmm_cache_bounds(cache, 0, batch, s["tokens"], _stream())
    return s["bounds"]


def _own_score(s):
    c, t, width = s["case"], s["tokens"], s["table"].shape[1]
    sp, cache, batch = _described(s)
    how = sp.make_select(c["qh"], 1, 0, 0, True, c["window"])
    scores = torch.empty((t, c["kvh"], width), device="cuda")
    sp.spmm_cache_score(cache, 0, batch, s["q"], t, how, scores, width, _stream())
    return scores


def _own_select(s):
    c, t, width = s["case"], s["tokens"], s["table"].shape[1]
    sp, cache, batch = _described(s)
    how = sp.make_select(c["qh"], c["lists"], c["first"], c["last"], True, c["window"])
    lists = torch.empty((t, c["kvh"], c["lists"]), dtype=torch.int32, device="cuda")
    sp.spmm_cache_select(cache, batch, s["scores"], t, width, how, lists, _stream())
    return lists


def _own_attend(s):
    c, t = s["case"], s["tokens"]
    sp, cache, batch = _described(s)
    how = sp.make_attend(c["qh"], c["new"], c["dim"] ** -0.5, True, c["window"], "bf16")
    out = torch.empty((c["qh"] * c["dim"], t), dtype=torch.bfloat16, device="cuda")
    work = torch.empty(sp.spmm_selected_work_bytes(cache, t, how, c["lists"]), dtype=torch.uint8, device="cuda")
    sp.spmm_cache_attend_selected(cache, 0, batch, s["q"], t, how, s["lists"], c["lists"], out, t, work, _stream())
    return out


def _own_weigh(s):
    c, t = s["case"], s["tokens"]
    sp, cache, batch = _described(s)
    how = sp.make_weigh(c["qh"], c["new"], c["dim"] ** -0.5, True, c["window"], DECAY)
    work = torch.empty(sp.spmm_weigh_work_bytes(cache, batch, t, how), dtype=torch.uint8, device="cuda")
    sp.spmm_cache_weigh(cache, 0, batch, s["q"], t, how, work, _stream())
    return s["weight"]


def _own_evict(s):
    c = s["case"]
    sp, cache, _ = _described(s)
    how = sp.make_evict(c["first"], c["last"], c["keep"])
    kept = torch.empty((c["layers"], c["rows"], c["kvh"], c["keep"]), dtype=torch.int32, device="cuda")
    lens = torch.empty_like(s["kv_len"])
    sp.spmm_cache_evict(cache, s["table"], s["kv_len"], s["keep"], how, s["to"], lens, kept, _stream())
    return kept, lens, *_parts(s)


def _parts(s):
    """The pool: tokens are moved as they are, so 8-bit ones come back as they are held."""
    return tuple(s[n] for n in ("k", "v", "k_scale", "v_scale", "weight") if s[n] is not None)


def _plain_bounds(s):
    c, page = s["case"], s["case"]["page"]
    new, end = s["q_start"].diff().long(), s["kv_len"].long()
    most = _pages(c["new"], page) + 1       # pages that new tokens can lie in
    at = ((end - new) // page)[:, None] + torch.arange(most, device="cuda")
    there = (new > 0)[:, None] & (at * page < end[:, None])
    seq, slot = there.nonzero(as_tuple=True)
    at = at[seq, slot]
    ids = s["table"].long()[seq, at]
    x = s["k"][0, ids].float()      # [page][head][token][dim]
    if c["cache"] == "s8":
        x = x * s["k_scale"][0, ids][..., None]
    held = (at[:, None] * page + torch.arange(page, device="cuda") < end[seq][:, None])[:, None, :, None]
    odd = (held & ~torch.isfinite(x)).any(2)
    hi, lo = x.masked_fill(~held, -math.inf).amax(2), x.masked_fill(~held, math.inf).amin(2)
    both = torch.stack((hi, lo), 2).masked_fill(odd[:, :, None], math.nan)
    s["bounds"][0, ids] = both.to(torch.bfloat16)
    return s["bounds"]


def _padded(s):
    """Queries [sequence][head][query heads of it, new][dim], and where the new tokens stand."""
    c = s["case"]
    seq, at = _where(s)
    row = torch.arange(s["tokens"], device="cuda") - s["q_start"].long()[seq]
    q = torch.zeros((c["seqs"], c["new"], c["qh"], c["dim"]), device="cuda")
    q[seq, row] = s["q"].float()
    q = q.view(c["seqs"], c["new"], c["kvh"], -1, c["dim"]).permute(0, 2, 3, 1, 4).reshape(c["seqs"], c["kvh"], -1, c["dim"])
    place = torch.full((c["seqs"], c["new"]), -1, dtype=torch.int64, device="cuda")       # (a row without a token sees nothing)
    place[seq, row] = at
    return q, place, seq, row


def _plain_score(s):
    c = s["case"]
    q, place, seq, row = _padded(s)
    both = s["bounds"][0][s["table"].clamp(min=0).long()].float().permute(0, 2, 4, 3, 1)       # [sequence][head][dim][2][page]
    x = q.clamp(min=0) @ both[..., 0, :].contiguous() + q.clamp(max=0) @ both[..., 1, :].contiguous()
    x = x.view(c["seqs"], c["kvh"], -1, c["new"], x.shape[-1]).amax(2)
    lo, hi = _spans(s)
    page = torch.arange(x.shape[-1], device="cuda")
    hidden = (page < lo[:, None]) | (page > hi[:, None])
    return x[seq, :, row].masked_fill(hidden[:, None], -math.inf)


def _plain_select(s):
    return _chosen(s["case"], s["scores"], *_spans(s))


def _plain_attend(s):
    c, t, page = s["case"], s["tokens"], s["case"]["page"]
    seq, at = _where(s)
    lists = s["lists"].long()
    ids = s["table"].long()[seq[:, None, None], lists.clamp(min=0)]
    head = torch.arange(c["kvh"], device="cuda")[None, :, None]
    k, v = s["k"][0][ids, head].float(), s["v"][0][ids, head].float()      # [token][head][listed page][..]
    if c["cache"] == "s8":
        k *= s["k_scale"][0][ids, head][..., None]
        v *= s["v_scale"][0][ids, head][..., None, :]
    key = lists[..., None] * page + torch.arange(page, device="cuda")
    seen = (lists >= 0)[..., None] & (key <= at[:, None, None, None])
    if c["window"]:
        seen = seen & (key > (at - c["window"])[:, None, None, None])
    k = k.view(t, c["kvh"], -1, c["dim"])
    v = v.permute(0, 1, 2, 4, 3).reshape(t, c["kvh"], -1, c["dim"])
    score = (s["q"].float().view(t, c["kvh"], -1, c["dim"]) @ k.transpose(2, 3)).mul_(c["dim"] ** -0.5)
    score.masked_fill_(~seen.view(t, c["kvh"], 1, -1), -math.inf)
    score -= score.amax(-1, keepdim=True).clamp(min=-3e38)
    p = score.exp_()
    total = p.sum(-1, keepdim=True)
    o = (p @ v) / torch.where(total > 0, total, torch.ones_like(total))
    return o.reshape(t, -1).t().to(torch.bfloat16).contiguous()


def _plain_weigh(s):
    c, page = s["case"], s["case"]["page"]
    ids = s["table"].clamp(min=0).long()
    k = s["k"][0][ids].float()     # [sequence][page][head][token][dim]
    if c["cache"] == "s8":
        k *= s["k_scale"][0][ids][..., None]
    length = ids.shape[1] * page
    k = k.permute(0, 2, 1, 3, 4).reshape(c["seqs"], c["kvh"], length, c["dim"])
    q, place, _, _ = _padded(s)
    score = (q @ k.transpose(2, 3)).mul_(c["dim"] ** -0.5).view(c["seqs"], c["kvh"], -1, c["new"], length)
    key, end, new = torch.arange(length, device="cuda"), s["kv_len"].long()[:, None], s["q_start"].diff().long()[:, None]
    seen = key <= place[..., None]
    if c["window"]:
        seen = seen & (key > place[..., None] - c["window"])
    score.masked_fill_(~seen[:, None, None], -math.inf)
    score -= score.amax(-1, keepdim=True).clamp(min=-3e38)
    p = score.exp_()
    total = p.sum(-1, keepdim=True)
    got = (p / torch.where(total > 0, total, torch.ones_like(total))).sum((2, 3))      # [sequence][head][token]
    old = s["weight"][0][ids].permute(0, 2, 1, 3).reshape(got.shape)
    got += old.masked_fill_((key >= end - new)[:, None], 0) * DECAY
    seq, at = ((key < end) & (new > 0)).nonzero(as_tuple=True)
    s["weight"][0, ids[seq, at // page], :, at % page] = got[seq, :, at]
    return s["weight"]


def _plain_evict(s):
    c, page = s["case"], s["case"]["page"]
    ids, to, end = s["table"].clamp(min=0).long(), s["to"].clamp(min=0).long(), s["kv_len"].long()
    length = ids.shape[1] * page
    key = torch.arange(length, device="cuda")
    n = torch.minimum(end, s["keep"].long())
    n_first = n.clamp(max=c["first"])
    n_last = torch.minimum(n - n_first, torch.full_like(n, c["last"]))
    held = key < end[:, None]
    always = held & ((key < n_first[:, None]) | (key >= (end - n_last)[:, None]))
    w = s["weight"][:, ids].permute(0, 1, 3, 2, 4).reshape(c["layers"], c["rows"], c["kvh"], length)
    w = w.masked_fill(always[:, None], math.inf).masked_fill_(~held[:, None], -math.inf)
    most = min(c["keep"], length)
    best = torch.sort(w, dim=-1, descending=True, stable=True).indices[..., :most]
    there = (torch.arange(most, device="cuda") < n[:, None])[:, None]
    best = torch.where(there, best, length).sort(-1).values        # [layer][row][head][kept]
    layer, row, head, slot = (best < length).nonzero(as_tuple=True)
    src = best[layer, row, head, slot]
    p, o, p2, o2 = ids[row, src // page], src % page, to[row, slot // page], slot % page
    moved = [s["k"][layer, p, head, o], s["v"][layer, p, head, :, o]]
    moved += [s[x][layer, p, head, o] if s[x] is not None else None for x in ("k_scale", "v_scale", "weight")]
    s["k"][layer, p2, head, o2], s["v"][layer, p2, head, :, o2] = moved[0], moved[1]
    s["weight"][layer, p2, head, o2] = moved[4]
    if s["k_scale"] is not None:
        s["k_scale"][layer, p2, head, o2], s["v_scale"][layer, p2, head, o2] = moved[2], moved[3]
    kept = torch.full((*best.shape[:3], c["keep"]), -1, dtype=torch.int32, device="cuda")
    kept[..., :most] = torch.where(best < length, best, -1)
    return kept, n.to(torch.int32), *_parts(s)


_own = {"bounds": _own_bounds, "score": _own_score, "select": _own_select, "attend": _own_attend, "weigh": _own_weigh, "evict": _own_evict}
_plain = {"bounds": _plain_bounds, "score": _plain_score, "select": _plain_select, "attend": _plain_attend, "weigh": _plain_weigh, "evict": _plain_evict}


# ---- the definition, sequence by sequence or token by token, in 64 bits -----------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"bounds": _exact_bounds, "score": _exact_score, "select": _exact_select, "attend": _exact_attend, "weigh": _exact_weigh,
            "evict": _exact_evict}[case["kind"]](s)


def _rows(s, b, h, name, tokens):
    """Keys or values of a sequence's first tokens, [token][dim]."""
    ids = s["table"][b, : _pages(tokens, s["case"]["page"])].long()
    x = s[name][0, ids, h].double()
    x = x if name == "k" else x.transpose(1, 2)
    if s[name + "_scale"] is not None:
        x = x * s[name + "_scale"][0, ids, h].double()[..., None]
    return x.reshape(-1, s["case"]["dim"])[:tokens]


def _exact_bounds(s):
    c, page, out = s["case"], s["case"]["page"], s["bounds"].double()
    for b, (n, p) in enumerate(zip(*_lengths(c))):
        if n == 0:
            continue
        begin = p // page * page
        for h in range(c["kvh"]):
            x = _rows(s, b, h, "k", n + p)[begin:]
            whole = x.shape[0] // page
            ids = s["table"][b, begin // page : _pages(n + p, page)].long()
            y = x[: whole * page].view(whole, page, c["dim"])
            if whole:
                out[0, ids[:whole], h] = torch.stack((y.max(1).values, y.min(1).values), 1)
            if whole * page < x.shape[0]:
                out[0, ids[whole], h] = torch.stack((x[whole * page :].max(0).values, x[whole * page :].min(0).values))
    return out


def _exact_score(s):
    c, page, group = s["case"], s["case"]["page"], s["case"]["qh"] // s["case"]["kvh"]
    new, past = _lengths(c)
    if sum(n * _pages(n + p, page) for n, p in zip(new, past)) * c["qh"] * c["dim"] > 4e10:
        return None
    out, first = torch.full((s["tokens"], c["kvh"], s["table"].shape[1]), -math.inf, dtype=torch.float64, device="cuda"), 0
    for b, (n, p) in enumerate(zip(new, past)):
        ids = s["table"][b, : _pages(n + p, page)].long()
        for i in range(n):
            lo, hi = _seen(c, p + i)
            limits = s["bounds"][0, ids[lo : hi + 1]].double()[:, :, None]        # [page][head][1][2][dim]
            q = s["q"][first + i].double().view(1, c["kvh"], group, c["dim"])
            out[first + i, :, lo : hi + 1] = torch.where(q > 0, q * limits[..., 0, :], q * limits[..., 1, :]).sum(-1).amax(2).t()
        first += n
    return out


def _exact_select(s):
    return None     # (whole numbers, of values that are given)


def _exact_attend(s):
    c, page, group = s["case"], s["case"]["page"], s["case"]["qh"] // s["case"]["kvh"]
    new, past = _lengths(c)
    if s["tokens"] * c["kvh"] > 4200:
        return None
    out, lists, t = torch.zeros((c["qh"], c["dim"], s["tokens"]), dtype=torch.float64, device="cuda"), s["lists"].cpu(), 0
    for b, (n, p) in enumerate(zip(new, past)):
        kv = [(_rows(s, b, h, "k", n + p), _rows(s, b, h, "v", n + p)) for h in range(c["kvh"])] if n else []
        for i in range(n):
            for h, (k, v) in enumerate(kv):
                ids = lists[t, h]
                key = (ids[ids >= 0].long()[:, None] * page + torch.arange(page)).flatten()
                key = key[(key <= p + i) & ((key > p + i - c["window"]) if c["window"] else True)].cuda()
                y = s["q"][t, h * group : (h + 1) * group].double() @ k[key].t().contiguous() / math.sqrt(c["dim"])
                out[h * group : (h + 1) * group, :, t] = torch.softmax(y, 1) @ v[key]
            t += 1
    return out.reshape(-1, s["tokens"])


def _exact_weigh(s):
    c, page, group = s["case"], s["case"]["page"], s["case"]["qh"] // s["case"]["kvh"]
    new, past = _lengths(c)
    if c["qh"] * c["dim"] * sum(n * (n + p) for n, p in zip(new, past)) > 3e12:
        return None
    out, first = s["weight"].double(), 0
    for b, (n, p) in enumerate(zip(new, past)):
        if n == 0:
            continue
        key, place = torch.arange(n + p, device="cuda"), torch.arange(p, p + n, device="cuda")[:, None]
        hidden = key > place
        if c["window"]:
            hidden = hidden | (place - key >= c["window"])
        ids, off = s["table"][b].long()[key // page], key % page
        for h in range(c["kvh"]):
            k, w = _rows(s, b, h, "k", n + p), out[0, ids, h, off]
            w = torch.where(key < p, DECAY * w, 0.0)
            for j in range(group):
                y = s["q"][first : first + n, h * group + j].double() @ k.t().contiguous() / math.sqrt(c["dim"])
                w = w + torch.softmax(y.masked_fill(hidden, -math.inf), 1).sum(0)
            out[0, ids, h, off] = w
        first += n
    return out


def _exact_evict(s):
    c, page = s["case"], s["case"]["page"]
    lens, ns = _held(c)
    kept = torch.full((c["layers"], c["rows"], c["kvh"], c["keep"]), -1, dtype=torch.int32, device="cuda")
    parts, names = _parts(s), [n for n in ("k", "v", "k_scale", "v_scale", "weight") if s[n] is not None]
    for b, (n, m) in enumerate(zip(lens, ns)):
        first = min(c["first"], m)
        last = min(c["last"], m - first)
        for i in range(c["layers"]):
            for h in range(c["kvh"]):
                w = s["weight"][i, s["table"][b, : _pages(n, page)].long(), h].flatten()[first : n - last]
                best = torch.sort(w.cpu(), descending=True, stable=True).indices[: m - first - last] + first
                src = torch.cat((torch.arange(first), best.sort().values, torch.arange(n - last, n))).cuda()
                slot = torch.arange(m, device="cuda")
                kept[i, b, h, :m] = src.to(torch.int32)
                p, o, p2, o2 = s["table"][b].long()[src // page], src % page, s["to"][b].long()[slot // page], slot % page
                for name, x in zip(names, parts):
                    if name == "v":
                        x[i, p2, h, :, o2] = x[i, p, h, :, o]
                    else:
                        x[i, p2, h, o2] = x[i, p, h, o]
    return kept, _ints(ns), *(x.double() if x.is_floating_point() else x for x in parts)
