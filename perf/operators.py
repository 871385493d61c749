"""Workloads of the paged key/value cache and its attention, as a user of the library runs them.

Between the sparse projections of a decoder layer lie, in this order:
  append   the stacked Q/K/V projection's output (rows = features, tokens contiguous, as spmm_run writes it) becomes
           queries (a root-mean-square norm of each head, a rotation by position) and new keys and values in the pages of
           a cache;
  attend   the new tokens' queries against all that their sequences hold in the cache, softmax in between; the result is
           laid out like the projection's output, for the next one;
  fork     the next generation of a batch's sequences (beams that go on from the same parent, sequences that are cut,
           freed or given room): pages that end inside both are copied, whole ones are shared;
  compact  the pages in use move to the front of the pool.

Layouts: keys [layer][page][head][token][dim], values [layer][page][head][dim][token], one page table for all layers.
8-bit caches hold a scale for each token and head.  Head counts, head sizes and lengths are those of the BERT
configurations of `workloads/` (4, 12 and 16 heads of 64; sequences of 16 to 384 tokens; batches of up to 6144 tokens), and,
for decoders with shared key/value heads, 32 query heads on 8 of 128 with contexts up to 128 thousand tokens.

Fields: seqs, new (most new tokens of a sequence), past (most tokens before them), ragged (both spread over a quarter of the
range and up, one sequence in seven without a new token), qh, kvh, dim, page (tokens), cache ("bf16" | "s8"), x ("f32" | "s8"),
norm, rope ("half" | "pairs" | "none"), causal, window (0: none); for pages: layers, rows, len, beam, pages, used, moved.
"""
import math

import torch

own = False     # whether run() makes the framework's calls; otherwise it computes the plain form

EPS = 1e-6
X_SCALE = 0.03      # of 8-bit projections
LARGEST = {"append": 1.0e9, "attend": 5.0e11, "fork": 1.5e9, "compact": 1.5e9}      # bytes; attend: operations + 60 a byte


def _append(name, seqs, new, past, ragged, qh, kvh, dim, page, cache="bf16", x="f32", norm=True, rope="half"):
    return {"name": name, "kind": "append", "seqs": seqs, "new": new, "past": past, "ragged": ragged, "qh": qh, "kvh": kvh, "dim": dim,
            "page": page, "cache": cache, "x": x, "norm": norm, "rope": rope}


def _attend(name, seqs, new, past, ragged, qh, kvh, dim, page, cache="bf16", causal=True, window=0):
    return {"name": name, "kind": "attend", "seqs": seqs, "new": new, "past": past, "ragged": ragged, "qh": qh, "kvh": kvh, "dim": dim,
            "page": page, "cache": cache, "causal": causal, "window": window}


def _fork(name, rows, beam, len, layers, kvh, dim, page, pages, cache="bf16"):
    return {"name": name, "kind": "fork", "rows": rows, "beam": beam, "len": len, "layers": layers, "kvh": kvh, "dim": dim, "page": page,
            "pages": pages, "cache": cache}


def _compact(name, rows, pages, used, moved, layers, kvh, dim, page, cache="bf16"):
    return {"name": name, "kind": "compact", "rows": rows, "pages": pages, "used": used, "moved": moved, "layers": layers, "kvh": kvh,
            "dim": dim, "page": page, "cache": cache}


def listed():
    return [
        # one token each of a few conversations, small decoder: latency
        _append("append_8x1_h12", 8, 1, 300, False, 12, 12, 64, 16),
        # a step's chunk of prompts of many lengths, shared key/value heads
        _append("append_prompts_h32", 6, 1100, 500, True, 32, 8, 128, 64),
        # 8-bit projections into an 8-bit cache, pairs rotated, no norms (values of the cache come back as what they stand for)
        _append("append_s8_h16", 3, 384, 0, True, 16, 16, 64, 32, cache="s8", x="s8", norm=False, rope="pairs"),
        # one conversation's next token: latency
        _attend("attend_1x1_h16", 1, 1, 776, False, 16, 16, 64, 16),
        # a serving batch's next tokens, contexts of all lengths
        _attend("attend_64x1_ragged_h32", 64, 1, 8191, True, 32, 8, 128, 64),
        # a few long documents, 8-bit cache, two drafted tokens checked beside the next one
        _attend("attend_4x3_131k_s8", 4, 3, 131000, False, 32, 8, 128, 64, cache="s8"),
        # an encoder's batch 16 x 384, every token sees the whole of its sequence
        _attend("attend_encoder_16x384_h16", 16, 384, 0, True, 16, 16, 64, 64, causal=False),
        # prompts without a past
        _attend("attend_prompts_2x4097_h32", 2, 4097, 0, False, 32, 8, 128, 32),
        # a chunk of new tokens behind a long past, 8-bit cache, small pages
        _attend("attend_chunk_500_past_15k_s8", 1, 500, 15000, False, 32, 8, 128, 16, cache="s8"),
        # a beam's step: four sequences go on from two of them
        _fork("fork_4_beams", 4, 4, 203, 12, 12, 64, 16, 96),
        # a batch of beams, larger pages, all layers of a large model
        _fork("fork_64_rows", 64, 4, 1000, 24, 16, 64, 64, 640),
        # a pool after many sequences have come and gone
        _compact("compact_2048_pages", 96, 2048, 900, 500, 12, 12, 64, 32),
    ]


def draw(rng):
    def size(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    while True:
        kind = rng.choice(("append", "attend", "attend", "attend", "fork", "compact"))
        qh, kvh, dim = rng.choice(((4, 4, 64), (12, 12, 64), (16, 16, 64), (12, 4, 64), (16, 2, 64), (32, 8, 128), (16, 16, 128), (8, 1, 128), (10, 5, 80)))
        page = rng.choice((16, 32, 64, 128))
        cache = rng.choice(("bf16", "bf16", "s8"))
        if kind == "append":
            c = _append("", size(1, 64), size(1, 2048), rng.choice((0, size(1, 1000))), rng.random() < 0.5, qh, kvh, dim, page, cache,
                        rng.choice(("f32", "f32", "s8")), rng.random() < 0.7, rng.choice(("half", "half", "pairs", "none")))
        elif kind == "attend":
            few = rng.random() < 0.5
            c = _attend("", size(1, 64), size(1, 4) if few else size(5, 2048), size(1, 100000) if few else rng.choice((0, size(1, 20000))),
                        rng.random() < 0.5, qh, kvh, dim, page, cache, rng.random() < 0.8, rng.choice((0, 0, 0, size(17, 4096))))
        elif kind == "fork":
            beam = rng.choice((2, 4, 5, 8))
            rows, length = beam * size(1, 12), size(1, 2000)
            need = rows // beam * (length // page + beam * 3) + rows
            c = _fork("", rows, beam, length, rng.choice((4, 12, 24)), kvh, dim, page, need + size(1, 64), cache)
        else:
            pages = size(40, 2048)
            used = rng.randrange(pages // 4, 3 * pages // 4)
            c = _compact("", size(1, 128), pages, used, rng.randrange(1, min(used, pages - used) + 1), rng.choice((4, 12, 24)), kvh, dim, page, cache)
        del c["name"]
        pool = c["layers"] * c["pages"] * _page_bytes(c) if "layers" in c else 0
        if _cost(c) <= LARGEST[kind] and pool <= 4 << 30 and _plain_bytes(c) <= 24 << 30:
            return c


# ---- what a case is made of: the same for every seed --------------------------------------------------------------------------

def _lengths(c):
    """(new, past) tokens of each sequence."""
    if not c["ragged"]:
        return [c["new"]] * c["seqs"], [c["past"]] * c["seqs"]
    new, past = [], []
    for b in range(c["seqs"]):
        f, g = 1 - 0.75 * ((b * 0.618034) % 1), 1 - 0.75 * ((b * 0.754878) % 1)
        new.append(0 if b % 7 == 5 else max(1, int(c["new"] * f)))
        past.append(int(c["past"] * g))
    return new, past


def _page_bytes(c):
    """One layer's keys and values of a page, and their scales."""
    n = c["kvh"] * c["page"]
    return 2 * n * (c["dim"] * 2 if c["cache"] == "bf16" else c["dim"] + 4)


def _tails(c):
    """Pages that a fork copies: of each beam's half that goes on, the first child keeps the last page, the others copy it."""
    groups, children = c["rows"] // c["beam"], _children(c["beam"])
    return groups * sum(n - 1 for n in children if n) if c["len"] % c["page"] else 0


def _children(beam):
    """How many of a beam's next sequences go on from each of its present ones."""
    half = (beam + 1) // 2
    return [beam // half + (i < beam % half) for i in range(half)] + [0] * (beam - half)


def _visible(c, new, past):
    """Pairs of a query and a key that it sees, of one sequence."""
    if not c["causal"]:
        return new * (new + past) if not c["window"] else sum(min(new + past, new + past - max(0, past + i - c["window"] + 1)) for i in range(new))
    seen = (past + i + 1 for i in range(new))
    return sum(min(s, c["window"]) if c["window"] else s for s in seen)


def work(case):
    c = case
    if c["kind"] == "append":
        new, _ = _lengths(c)
        t, heads = sum(new), c["qh"] + 2 * c["kvh"]
        kv = 2 * c["kvh"] * t * (c["dim"] * 2 if c["cache"] == "bf16" else c["dim"] + 4)
        return {"bytes": t * heads * c["dim"] * (4 if c["x"] == "f32" else 1) + t * c["qh"] * c["dim"] * 2 + kv, "flops": 10 * t * heads * c["dim"]}
    if c["kind"] == "attend":
        new, past = _lengths(c)
        pairs = sum(_visible(c, n, p) for n, p in zip(new, past))
        seen = 0
        for n, p in zip(new, past):     # keys that some query of the sequence sees
            seen += 0 if not n else n + p if not c["window"] else min(n + p, n + c["window"] - 1) if c["causal"] else min(n + p, n + p - max(0, p - c["window"] + 1))
        kv = 2 * c["kvh"] * seen * (c["dim"] * 2 if c["cache"] == "bf16" else c["dim"] + 4)
        return {"bytes": kv + sum(new) * c["qh"] * c["dim"] * 4, "flops": 4 * pairs * c["qh"] * c["dim"]}
    copied = _tails(c) if c["kind"] == "fork" else c["moved"]
    width = -(-(c["len"] + 1) // c["page"]) if c["kind"] == "fork" else -(-c["used"] // c["rows"])
    return {"bytes": 2 * copied * c["layers"] * _page_bytes(c) + 8 * c["rows"] * width, "flops": 0}


def _cost(c):
    w = work(c)
    return w["flops"] + 60 * w["bytes"] if c["kind"] == "attend" else w["bytes"]


def _plain_bytes(c):
    """Memory that the plain form of attention takes: scores and widened keys and values."""
    if c["kind"] != "attend":
        return 0
    most = c["new"] + c["past"]
    return c["seqs"] * most * (8 * c["qh"] * c["new"] + 12 * c["kvh"] * c["dim"])


# ---- inputs -------------------------------------------------------------------------------------------------------------------

def _pool(c, layers, pages, g):
    """A cache's pages: keys, values, and their scales where they are held in 8 bits."""
    shape = (layers, pages, c["kvh"])
    k_shape, v_shape = (*shape, c["page"], c["dim"]), (*shape, c["dim"], c["page"])
    if c["cache"] == "s8":
        k, v = (torch.randint(-127, 128, s, generator=g, device="cuda", dtype=torch.int8) for s in (k_shape, v_shape))
        ks, vs = (torch.rand((*shape, c["page"]), generator=g, device="cuda") * 0.012 + 0.01 for _ in range(2))
        return {"k": k, "v": v, "k_scale": ks, "v_scale": vs}
    k, v = (torch.randn(s, generator=g, device="cuda", dtype=torch.bfloat16) for s in (k_shape, v_shape))
    return {"k": k, "v": v, "k_scale": None, "v_scale": None}


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    c, g = case, torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": c}
    if c["kind"] in ("append", "attend"):
        new, past = _lengths(c)
        held = [-(-(n + p) // c["page"]) for n, p in zip(new, past)]
        pages, width = sum(held) + 2, max(max(held), 1)
        s |= _pool(c, 1, pages, g)
        order = torch.randperm(pages, generator=g, device="cuda")[: sum(held)].to(torch.int32).cpu()
        table, at = torch.full((len(held), width), -1, dtype=torch.int32), 0
        for b, n in enumerate(held):
            table[b, :n] = order[at : at + n]
            at += n
        start = [0]
        for n in new:
            start.append(start[-1] + n)
        t = start[-1]
        s |= {"table": table.cuda(), "q_start": _ints(start), "kv_len": _ints([n + p for n, p in zip(new, past)]), "tokens": t}
        if c["kind"] == "append":
            features = (c["qh"] + 2 * c["kvh"]) * c["dim"]
            x = torch.randn((features, t), generator=g, device="cuda")
            s["x"] = (x * 32).round().clamp(-127, 127).to(torch.int8) if c["x"] == "s8" else x
            s["q_weight"], s["k_weight"] = (torch.rand(c["dim"], generator=g, device="cuda") + 0.5 if c["norm"] else None for _ in range(2))
            s["rope"] = None
            if c["rope"] != "none":
                turn = torch.arange(c["new"] + c["past"], device="cuda", dtype=torch.float64)[:, None]
                turn = turn * 10000.0 ** (-torch.arange(0, c["dim"], 2, device="cuda", dtype=torch.float64) / c["dim"])
                s["rope"] = torch.stack((turn.cos(), turn.sin()), dim=-1).float()      # [position][pair][cos, sin]
        else:
            s["q"] = (torch.randn((t, c["qh"], c["dim"]), generator=g, device="cuda") * 1.5).to(torch.bfloat16)
        return s
    s |= _pool(c, c["layers"], c["pages"], g)
    order = torch.randperm(c["pages"], generator=g, device="cuda").to(torch.int32).cpu()
    rows = c["rows"]
    if c["kind"] == "fork":
        # the rows of a beam share their prompt's whole pages; the last page, or two, are each row's own
        whole, width = c["len"] // c["page"], -(-(c["len"] + 1) // c["page"])
        table, at = torch.full((rows, width + 1), -1, dtype=torch.int32), 0
        for r in range(rows):
            first, shared = r - r % c["beam"], max(0, whole - 1)
            if r == first:
                table[r, :shared] = order[at : at + shared]
                at += shared
            table[r, :shared] = table[first, :shared]
            mine = -(-c["len"] // c["page"]) - shared
            table[r, shared : shared + mine] = order[at : at + mine]
            at += mine
        parent, children = [], _children(c["beam"])
        pick = torch.rand((rows // c["beam"], c["beam"]), generator=g, device="cuda").argsort(dim=1).cpu().tolist()
        for q, group in enumerate(pick):
            parent += [q * c["beam"] + group[i] for i, n in enumerate(children) for _ in range(n)]
        s |= {"table": table.cuda(), "kv_len": _ints([c["len"]] * rows), "parent": _ints(parent), "keep": _ints([c["len"]] * rows),
              "want": _ints([c["len"] + 1] * rows)}
    else:
        # `moved` of the pages in use lie behind the first `used` pages of the pool
        low, high = torch.randperm(c["used"], generator=g, device="cuda").cpu(), torch.randperm(c["pages"] - c["used"], generator=g, device="cuda").cpu()
        ids = torch.cat((low[: c["used"] - c["moved"]], high[: c["moved"]] + c["used"])).to(torch.int32)
        ids = ids[torch.randperm(c["used"], generator=g, device="cuda").cpu()]
        width = -(-c["used"] // rows)
        table = torch.full((rows * width,), -1, dtype=torch.int32)
        table[: c["used"]] = ids
        s["table"] = table.reshape(rows, width).cuda()
    return s


# ---- one pass -----------------------------------------------------------------------------------------------------------------

def run(state):
    return (_own if own else _plain)[state["case"]["kind"]](state)


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _values(s):
    """An 8-bit cache as the values it stands for."""
    if s["k_scale"] is None:
        return s["k"], s["v"]
    return (s["k"] * s["k_scale"][..., None]).to(torch.bfloat16), (s["v"] * s["v_scale"][..., None, :]).to(torch.bfloat16)


def _own_append(s):
    import paper_2306_16601_amd as sp
    c, t = s["case"], s["tokens"]
    cache = sp.make_cache(s["k"], s["v"], s["k_scale"], s["v_scale"])
    batch = sp.make_batch(s["q_start"], s["kv_len"], s["table"])
    how = sp.make_append(c["qh"], c["x"], X_SCALE if c["x"] == "s8" else 1.0, 0, s["q_weight"], s["k_weight"], EPS, s["rope"], c["rope"] == "pairs")
    q = torch.empty((t, c["qh"], c["dim"]), dtype=torch.bfloat16, device="cuda")
    sp.spmm_cache_append(cache, 0, batch, s["x"], t, t, how, q, _stream())
    return (q, *_values(s))


def _own_attend(s):
    import paper_2306_16601_amd as sp
    c, t = s["case"], s["tokens"]
    cache = sp.make_cache(s["k"], s["v"], s["k_scale"], s["v_scale"])
    batch = sp.make_batch(s["q_start"], s["kv_len"], s["table"])
    how = sp.make_attend(c["qh"], c["new"], c["dim"] ** -0.5, c["causal"], c["window"], "bf16")
    out = torch.empty((c["qh"] * c["dim"], t), dtype=torch.bfloat16, device="cuda")
    work = torch.empty(sp.spmm_attend_work_bytes(cache, c["seqs"], t, how), dtype=torch.uint8, device="cuda")
    sp.spmm_cache_attend(cache, 0, batch, s["q"], t, how, out, t, work, _stream())
    return out


def _own_fork(s):
    import paper_2306_16601_amd as sp
    cache = sp.make_cache(s["k"], s["v"], s["k_scale"], s["v_scale"])
    table, kv_len = torch.empty_like(s["table"]), torch.empty_like(s["kv_len"])
    info = torch.empty(4, dtype=torch.int32, device="cuda")
    work = torch.empty(sp.spmm_cache_work_bytes(cache, s["case"]["rows"]), dtype=torch.uint8, device="cuda")
    sp.spmm_cache_fork(cache, s["table"], s["kv_len"], s["parent"], s["keep"], s["want"], table, kv_len, info, work, _stream())
    return table, kv_len, info[:3], *_pages(s)


def _own_compact(s):
    import paper_2306_16601_amd as sp
    cache = sp.make_cache(s["k"], s["v"], s["k_scale"], s["v_scale"])
    table, info = torch.empty_like(s["table"]), torch.empty(4, dtype=torch.int32, device="cuda")
    work = torch.empty(sp.spmm_cache_work_bytes(cache, s["case"]["rows"]), dtype=torch.uint8, device="cuda")
    sp.spmm_cache_compact(cache, s["table"], table, info, work, _stream())
    return table, info[:3], *_pages(s)


def _pages(s):
    """The pool: pages are moved as they are, so 8-bit ones come back as they are held."""
    return tuple(s[n] for n in ("k", "v", "k_scale", "v_scale") if s[n] is not None)


def _where(s):
    """Of each new token: its sequence, its place in it, and its page."""
    t = torch.arange(s["tokens"], device="cuda")
    start = s["q_start"].long()
    seq = torch.searchsorted(start[1:], t, right=True)
    at = s["kv_len"].long()[seq] - start[seq + 1] + t
    return seq, at, s["table"][seq, at // s["case"]["page"]].long()


def _plain_append(s):
    c, t = s["case"], s["tokens"]
    x = s["x"].float() * X_SCALE if c["x"] == "s8" else s["x"]
    x = x.view(-1, c["dim"], t).permute(2, 0, 1)       # [token][head][dim]
    q, k, v = x[:, : c["qh"]], x[:, c["qh"] : c["qh"] + c["kvh"]], x[:, c["qh"] + c["kvh"] :]
    seq, at, page = _where(s)
    if c["norm"]:
        q = q * (q.square().mean(-1, keepdim=True) + EPS).rsqrt() * s["q_weight"]
        k = k * (k.square().mean(-1, keepdim=True) + EPS).rsqrt() * s["k_weight"]
    if c["rope"] != "none":
        cos, sin = s["rope"][at][:, None, :, 0], s["rope"][at][:, None, :, 1]
        q, k = _turned(q, cos, sin, c["rope"]), _turned(k, cos, sin, c["rope"])
    off = at % c["page"]
    if c["cache"] == "s8":
        k, ks = _eight(k)
        v, vs = _eight(v)
        s["k_scale"][0, page, :, off], s["v_scale"][0, page, :, off] = ks, vs
    s["k"][0, page, :, off] = k.to(s["k"].dtype)
    s["v"][0, page, :, :, off] = v.to(s["v"].dtype)
    return (q.to(torch.bfloat16).contiguous(), *_values(s))


def _turned(x, cos, sin, rope):
    if rope == "half":
        a, b = x.chunk(2, dim=-1)
        return torch.cat((a * cos - b * sin, b * cos + a * sin), dim=-1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack((a * cos - b * sin, b * cos + a * sin), dim=-1).flatten(-2)


def _eight(x):
    """Codes of 8 bits, the largest of a token's head at 127, and their scales."""
    most = x.abs().amax(-1)
    return (x * torch.where(most > 0, 127.0 / most, torch.zeros_like(most))[..., None]).round(), most / 127.0


def _plain_attend(s):
    c, t = s["case"], s["tokens"]
    seqs, group, new = c["seqs"], c["qh"] // c["kvh"], c["new"]
    k, v = s["k"][0], s["v"][0]
    pages = s["table"].clamp(min=0).long()
    length = pages.shape[1] * c["page"]
    k = k[pages].permute(0, 2, 1, 3, 4).reshape(seqs, c["kvh"], length, c["dim"]).float()
    v = v[pages].permute(0, 2, 1, 4, 3).reshape(seqs, c["kvh"], length, c["dim"]).float()
    if c["cache"] == "s8":
        k *= s["k_scale"][0][pages].permute(0, 2, 1, 3).reshape(seqs, c["kvh"], length, 1)
        v *= s["v_scale"][0][pages].permute(0, 2, 1, 3).reshape(seqs, c["kvh"], length, 1)
    seq, at, _ = _where(s)
    row = torch.arange(t, device="cuda") - s["q_start"].long()[seq]
    q = torch.zeros((seqs, new, c["qh"], c["dim"]), device="cuda")
    q[seq, row] = s["q"].float()
    q = q.view(seqs, new, c["kvh"], group, c["dim"]).permute(0, 2, 3, 1, 4).reshape(seqs, c["kvh"], group * new, c["dim"])
    place = torch.full((seqs, new), -1, dtype=torch.int64, device="cuda")       # (a row without a token sees nothing)
    place[seq, row] = at
    key = torch.arange(length, device="cuda")
    seen = key < s["kv_len"].long()[:, None, None]
    if c["causal"]:
        seen = seen & (key <= place[..., None])
    if c["window"]:
        seen = seen & (key > place[..., None] - c["window"])
    seen = (seen & (place[..., None] >= 0))[:, None, None]
    score = (q @ k.transpose(2, 3)).mul_(c["dim"] ** -0.5).view(seqs, c["kvh"], group, new, length)
    score.masked_fill_(~seen, -math.inf)
    score -= score.amax(-1, keepdim=True).clamp(min=-3e38)
    p = score.exp_()
    total = p.sum(-1, keepdim=True)
    o = (p.view(seqs, c["kvh"], group * new, length) @ v).view(seqs, c["kvh"], group, new, c["dim"]) / torch.where(total > 0, total, torch.ones_like(total))
    o = o.permute(0, 3, 1, 2, 4).reshape(seqs, new, c["qh"] * c["dim"])[seq, row]
    return o.t().to(torch.bfloat16).contiguous()


def _moved(s, src, dst, move):
    """Copies the pages of all layers where `move`."""
    for x in _pages(s):
        x[:, dst[move]] = x[:, src[move]]


def _plain_fork(s):
    c, page, pages = s["case"], s["case"]["page"], s["case"]["pages"]
    old, width = s["table"].long(), s["table"].shape[1]
    parent, row, i = s["parent"].long(), torch.arange(s["parent"].numel(), device="cuda")[:, None], torch.arange(width, device="cuda")
    kept = torch.where(parent >= 0, torch.minimum(s["keep"].long(), s["kv_len"].long()[parent.clamp(min=0)]), 0)
    room = torch.maximum(kept, s["want"].long())
    ref = old[parent.clamp(min=0)]
    whole, tail = i < (kept // page)[:, None], (i == (kept // page)[:, None]) & (kept % page > 0)[:, None]
    none = pages        # (the number of a page that is not there)
    used = torch.zeros(pages + 1, dtype=torch.bool, device="cuda")
    used[torch.where(old >= 0, old, none).flatten()] = True
    shared = torch.zeros(pages + 1, dtype=torch.bool, device="cuda")
    shared[torch.where(whole, ref, none).flatten()] = True
    first = torch.full((pages + 1,), 1 << 30, device="cuda")
    at = torch.where(tail, ref, none)
    first.scatter_reduce_(0, at.flatten(), row.expand_as(at).flatten(), "amin")
    stays = tail & (first[at] == row) & ~shared[at]
    fresh = (tail & ~stays) | ((i >= (-(-kept // page))[:, None]) & (i < (-(-room // page))[:, None]))
    free = torch.argsort(used[:pages].to(torch.int8), stable=True)     # the lowest free pages first
    rank = fresh.flatten().long().cumsum(0).view_as(fresh) - 1
    got = free[rank.clamp(min=0, max=pages - 1)]
    table = torch.where(whole | stays, ref, torch.where(fresh, got, -1))
    _moved(s, ref, got, tail & ~stays)
    left = torch.zeros(pages + 1, dtype=torch.bool, device="cuda")
    left[torch.where(table >= 0, table, none).flatten()] = True
    need = fresh.sum() - (pages - used[:pages].sum())
    info = torch.stack((need.clamp(min=0), (tail & ~stays).sum(), left[:pages].sum()))
    return table.to(torch.int32), kept.to(torch.int32), info.to(torch.int32), *_pages(s)


def _plain_compact(s):
    pages, old = s["case"]["pages"], s["table"].long()
    used = torch.zeros(pages + 1, dtype=torch.bool, device="cuda")
    used[torch.where(old >= 0, old, pages).flatten()] = True
    used = used[:pages]
    front = torch.arange(pages, device="cuda") < used.sum()
    hole, late = front & ~used, ~front & used
    free = torch.argsort((~hole).to(torch.int8), stable=True)      # the holes first, in order
    to = torch.where(late, free[(late.long().cumsum(0) - 1).clamp(min=0)], torch.arange(pages, device="cuda"))
    table = torch.where(old >= 0, to[old.clamp(min=0)], -1)
    _moved(s, torch.arange(pages, device="cuda"), to, late)
    info = torch.stack((torch.zeros_like(late.sum()), late.sum(), used.sum()))
    return table.to(torch.int32), info.to(torch.int32), *_pages(s)


_own = {"append": _own_append, "attend": _own_attend, "fork": _own_fork, "compact": _own_compact}
_plain = {"append": _plain_append, "attend": _plain_attend, "fork": _plain_fork, "compact": _plain_compact}


# ---- the definition, token by token or page by page, in 64 bits ---------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "fork": _exact_fork, "compact": _exact_compact}[case["kind"]](s)


def _exact_append(s):
    c = s["case"]
    x = s["x"].double().t() * (X_SCALE if c["x"] == "s8" else 1.0)      # [token][feature]
    new, past = _lengths(c)
    k, v = s["k"].double(), s["v"].double()
    if c["cache"] == "s8":
        k, v = k * s["k_scale"].double()[..., None], v * s["v_scale"].double()[..., None, :]
    angle = 10000.0 ** (-torch.arange(0, c["dim"], 2, dtype=torch.float64, device="cuda") / c["dim"])
    qs, first = [], 0
    for b, (n, p) in enumerate(zip(new, past)):
        heads = [x[first : first + n, h * c["dim"] : (h + 1) * c["dim"]].clone() for h in range(c["qh"] + 2 * c["kvh"])]
        place = torch.arange(p, p + n, device="cuda")
        for h in range(c["qh"] + c["kvh"]):
            y = heads[h]
            if c["norm"]:
                y = y / torch.sqrt((y * y).sum(1) / c["dim"] + EPS)[:, None] * s["q_weight" if h < c["qh"] else "k_weight"].double()
            if c["rope"] != "none":
                turn = torch.polar(torch.ones(n, c["dim"] // 2, dtype=torch.float64, device="cuda"), place[:, None] * angle)
                both = (y[:, : c["dim"] // 2], y[:, c["dim"] // 2 :]) if c["rope"] == "half" else (y[:, ::2], y[:, 1::2])
                z = torch.complex(*(t.contiguous() for t in both)) * turn
                y = torch.cat((z.real, z.imag), 1) if c["rope"] == "half" else torch.view_as_real(z).reshape(n, -1)
            heads[h] = y
        pages, off = s["table"][b].long()[place // c["page"]], place % c["page"]
        for h in range(c["kvh"]):
            k[0, pages, h, off] = heads[c["qh"] + h]
            v[0, pages, h, :, off] = heads[c["qh"] + c["kvh"] + h]
        qs.append(torch.stack(heads[: c["qh"]], 1))
        first += n
    return torch.cat(qs), k, v


def _exact_attend(s):
    c = s["case"]
    new, past = _lengths(c)
    if c["qh"] * c["dim"] * sum(n * (n + p) for n, p in zip(new, past)) > 3e12:
        return None
    out, first = torch.zeros((c["qh"], c["dim"], s["tokens"]), dtype=torch.float64, device="cuda"), 0
    group = c["qh"] // c["kvh"]
    for b, (n, p) in enumerate(zip(new, past)):
        if n == 0:
            continue
        ids = s["table"][b, : -(-(n + p) // c["page"])].long()
        key, place = torch.arange(n + p, device="cuda"), torch.arange(p, p + n, device="cuda")[:, None]
        hidden = (key > place) if c["causal"] else torch.zeros((n, n + p), dtype=torch.bool, device="cuda")
        if c["window"]:
            hidden = hidden | (place - key >= c["window"])
        for h in range(c["kvh"]):
            k, v = s["k"][0, ids, h].double(), s["v"][0, ids, h].double()
            if c["cache"] == "s8":
                k, v = k * s["k_scale"][0, ids, h].double()[:, :, None], v * s["v_scale"][0, ids, h].double()[:, None, :]
            k, v = k.reshape(-1, c["dim"])[: n + p], v.transpose(1, 2).reshape(-1, c["dim"])[: n + p]
            for j in range(group):
                y = s["q"][first : first + n, h * group + j].double() @ k.t().contiguous() / math.sqrt(c["dim"])
                out[h * group + j, :, first : first + n] = (torch.softmax(y.masked_fill(hidden, -math.inf), 1) @ v).t()
        first += n
    return out.reshape(-1, s["tokens"])


def _exact_fork(s):
    c, page = s["case"], s["case"]["page"]
    old, lens = s["table"].tolist(), s["kv_len"].tolist()
    parent, keep, want = (s[n].tolist() for n in ("parent", "keep", "want"))
    in_use = {p for row in old for p in row if p >= 0}
    free = sorted(set(range(c["pages"])) - in_use)
    kept = [min(k, lens[p]) if p >= 0 else 0 for p, k in zip(parent, keep)]
    shared = {old[p][i] for p, k in zip(parent, kept) if p >= 0 for i in range(k // page)}
    table, taken, copies = [], set(), []
    for p, k, w in zip(parent, kept, want):
        row = old[p][: k // page] if p >= 0 else []
        if k % page:
            last = old[p][k // page]
            if last in shared or last in taken:
                copies.append((last, free[0]))
                row.append(free.pop(0))
            else:
                row.append(last)
            taken.add(last)
        while len(row) * page < max(k, w):
            row.append(free.pop(0))
        table.append(row + [-1] * (len(old[0]) - len(row)))
    left = {p for row in table for p in row if p >= 0}
    return _ints(table), _ints(kept), _ints([0, len(copies), len(left)]), *_exact_pages(s, copies)


def _exact_compact(s):
    old = s["table"].tolist()
    used = sorted({p for row in old for p in row if p >= 0})
    holes = sorted(set(range(len(used))) - set(used))
    moves = list(zip([p for p in used if p >= len(used)], holes))
    to = dict(moves)
    return _ints([[to.get(p, p) for p in row] for row in old]), _ints([0, len(moves), len(used)]), *_exact_pages(s, moves)


def _exact_pages(s, moves):
    pools = _pages(s)
    for src, dst in moves:
        for x in pools:
            x[:, dst] = x[:, src]
    return tuple(x.double() if x.is_floating_point() else x for x in pools)
