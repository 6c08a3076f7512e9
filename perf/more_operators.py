"""Attention over whole prompts and the pages of the cache that keeps them, as measurable cases.

A program that serves prompts takes a batch of them, of different lengths and packed one behind another, through

  prompt   every token attends to its own sequence, up to itself (causal) or to all of it: grouped heads, any lengths.

and keeps their keys and values in pages of a pool.  Which sequence holds which page is a table; a page may belong to several
sequences and is counted, one count a holder.  Between its steps such a program calls

  fork     every row of the next table takes the first tokens of a row of the last one and room for more: it shares the
           pages that these tokens fill, gets its own copy of a page that they fill in part, and fresh pages behind; what
           nobody holds any more is free.  Going on, cutting back, continuing one sequence in several ways and ending
           one are all this call.  Fresh pages are the free ones with the lowest numbers, row by row.
  compact  the pages in use go to the lowest numbers of the pool, the tables with them.
  copy     pages of one cache to pages of another (the cache of the prompts to the one of the answers), whose tokens
           may lie in another order.

Tables and counts of a step are new tensors; the caches are written in place.  q, k, v are [heads, tokens, head_dim] views, a
cache is [pages, heads, page, head_dim], any strides.
"""
import math

import numpy
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}

PROMPT = dict(op="prompt", batch=1, len_min=1, len_max=1, q_heads=32, kv_heads=8, head_dim=128, dtype="bf16", causal=True, order="nhd")
POOL = dict(page=16, kv_heads=8, head_dim=128, dtype="bf16", cache="hnd")
FORK = dict(POOL, op="fork", batch=16, len_min=1, len_max=1000, mode="step", room=1, width=1, prefix=0, spare=0.1)
COMPACT = dict(POOL, op="compact", batch=16, len_min=1, len_max=1000, prefix=0, used=0.5)
COPY = dict(POOL, op="copy", pages=7, pool=64, to_cache="hnd")


def listed():
    return [
        # the smallest: one short prompt in front of a clip, few heads
        dict(PROMPT, name="prompt_short", len_min=77, len_max=77, q_heads=8, kv_heads=2, head_dim=64),
        # an ordinary batch: sixteen prompts of 20 to 2,000 tokens
        dict(PROMPT, name="prompt_batch", batch=16, len_min=20, len_max=2000),
        # many short requests, fp16, seven query heads a key head, head_dim 64
        dict(PROMPT, name="prompt_ragged", batch=150, len_min=1, len_max=700, q_heads=28, kv_heads=4, head_dim=64, dtype="fp16"),
        # the frames of a clip, each attending to itself, as many key heads as query heads, head by head in memory
        dict(PROMPT, name="prompt_frames", batch=6, len_min=1560, len_max=1560, q_heads=40, kv_heads=40, causal=False, order="hnd"),
        # a document as long as a 480p clip: the largest
        dict(PROMPT, name="prompt_long", len_min=32760, len_max=32760, q_heads=32, kv_heads=8),
        # decoding goes on: each of 16 sequences gets room for one more token
        dict(FORK, name="fork_step", mode="step"),
        # eight questions continued in eight ways each, large pages that are copied where they are filled in part
        dict(FORK, name="fork_beams", batch=64, len_min=200, len_max=4000, page=128, mode="beams", width=8, room=130, cache="nhd", prefix=1000),
        # turnover of a large pool: a quarter of 512 sequences ends, some are forked, drafts are cut back, the others grow
        dict(FORK, name="fork_turnover", batch=512, len_max=8000, kv_heads=1, head_dim=64, mode="turnover", room=600, dtype="fp16"),
        # a small pool, three fifths in use
        dict(COMPACT, name="compact_few", batch=9, len_max=600, used=0.6),
        # half of a pool of large pages, five of a clip's heads
        dict(COMPACT, name="compact_frames", batch=40, len_min=1000, len_max=6000, page=128, kv_heads=5, prefix=32760, cache="nhd"),
        # a finished prompt's few pages
        dict(COPY, name="copy_few", pages=7),
        # the pages of a 480p clip with 40 heads, from head-major into token-major pages
        dict(COPY, name="copy_clip", pages=512, pool=700, page=64, kv_heads=40, to_cache="nhd"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: any operator, length, head layout, page, type and way of forking of the ranges above."""
    op = rng.choice(["prompt", "prompt", "fork", "fork", "compact", "copy"])
    if op == "prompt":
        kv = rng.choice([1, 2, 4, 5, 8, 10, 40])
        case = dict(PROMPT, q_heads=kv * rng.choice([1, 2, 3, 4, 5, 7, 8]) if kv < 40 else 40, kv_heads=kv, head_dim=rng.choice([64, 128, 128]),
                    dtype=rng.choice(["bf16", "bf16", "fp16"]), causal=rng.random() < 0.8, order=rng.choice(["hnd", "nhd", "nhd"]))
        case["batch"] = _log(rng, 1, 300)
        case["len_max"] = _log(rng, 1, min(32760, 200000 // case["batch"]))
        case["len_min"] = rng.choice([1, case["len_max"], _log(rng, 1, case["len_max"])])
        while work(case)["flops"] > 8e12:
            case["len_max"] = case["len_max"] * 2 // 3
            case["len_min"] = min(case["len_min"], case["len_max"])
        return case
    pool = dict(page=rng.choice([16, 16, 32, 64, 128, 256]), kv_heads=rng.choice([1, 2, 4, 5, 8]), head_dim=rng.choice([64, 96, 128, 128]),
                dtype=rng.choice(["bf16", "bf16", "fp16"]), cache=rng.choice(["hnd", "nhd"]))
    token = pool["kv_heads"] * pool["head_dim"] * 2                       # bytes of a token's keys
    if op == "copy":
        pages = _log(rng, 1, min(20000, (1 << 28) // (token * pool["page"])))
        return dict(COPY, **pool, pages=pages, pool=pages + _log(rng, 1, pages + 1), to_cache=rng.choice(["hnd", "nhd"]))
    most = (1 << 28) // token                                             # tokens of all sequences
    batch = _log(rng, 1, 500)
    case = dict(batch=batch, len_max=max(1, min(_log(rng, 1, 8000), most // batch)), prefix=rng.choice([0, 0, _log(rng, 1, 4000)]))
    case["len_min"] = rng.choice([1, case["len_max"], _log(rng, 1, case["len_max"])])
    if op == "compact":
        return dict(COMPACT, **pool, **case, used=rng.uniform(0.2, 0.95))
    return dict(FORK, **pool, **case, mode=rng.choice(["step", "beams", "turnover"]), width=_log(rng, 1, 16), room=_log(rng, 1, 300),
                spare=rng.uniform(0.0, 0.5))


# ------------------------------------------------------------------ what a program has in hand

def _spread(n, lo, hi, step=0.7548776662466927):
    """n whole numbers from lo to hi, unlike their neighbours, both ends among them."""
    return [hi if b == 0 else lo if b == n - 1 else lo + int((b * step) % 1.0 * (hi - lo + 1)) for b in range(n)]


def _up(n, page):
    return -(-n // page)


def _rows(c):
    """The rows of a pool's table: tokens each holds, first pages it has in common with its group, which pages those are.
    Pages are numbered in the order they were given out: the shared prefix's, then row by row."""
    lens = numpy.array(_spread(c["batch"], c["len_min"], c["len_max"]))
    width = c["width"] if c.get("mode") == "beams" else 1
    given = _up(c["prefix"], c["page"])
    table = numpy.zeros((c["batch"], int(_up(lens.max(), c["page"]))), dtype=numpy.int64)
    for first in range(0, c["batch"], width):
        group = range(first, min(first + width, c["batch"]))
        common = int(lens[list(group)].min()) // c["page"] // 2 if width > 1 else 0
        table[list(group), :common] = given + numpy.arange(common)
        given += common
        for b in group:
            n = int(_up(lens[b], c["page"]))
            table[b, common:n] = given + numpy.arange(n - common)
            given += n - common
    return lens, table, given


def _wishes(c, lens):
    """parent, tokens kept and room of every row of the next table."""
    B = c["batch"]
    parent, room = numpy.arange(B), numpy.array(_spread(B, 1, c["room"], 0.6180339887498949))
    keep = lens.copy()
    if c["mode"] == "beams":       # every group goes on from two of its rows
        group = parent // c["width"] * c["width"]
        parent = numpy.minimum(group + numpy.where(parent % 3 == 0, 0, c["width"] // 2), B - 1)
        keep = lens[parent]
    elif c["mode"] == "turnover":
        b = numpy.arange(B)
        parent = numpy.where(b % 4 == 3, -1, numpy.where(b % 7 == 2, (b * 5 + 1) % B, b))
        keep = numpy.maximum(lens[numpy.maximum(parent, 0)] - b % 5, 0)
    return parent, keep, keep + room


def _counts(table, lens, page, n_pages, prefix):
    counts = numpy.zeros(n_pages, dtype=numpy.int64)
    counts[:prefix] = 1
    held = numpy.arange(table.shape[1]) < _up(lens, page)[:, None]
    return counts + numpy.bincount(table[held], minlength=n_pages)


def _cache(g, c, pages, order):
    """[pages, heads, page, head_dim], the page's tokens outermost in memory for "nhd"."""
    H, P, D = c["kv_heads"], c["page"], c["head_dim"]
    x = torch.empty((pages, P, H, D) if order == "nhd" else (pages, H, P, D), dtype=DTYPES[c["dtype"]], device="cuda").normal_(generator=g)
    return x.transpose(1, 2) if order == "nhd" else x


def _cuda(x):
    return torch.from_numpy(numpy.ascontiguousarray(x)).to(torch.int32).cuda()


def _pool(c):
    """lens, table, pages given out, pages of the pool, and for a fork the rows of the next table"""
    lens, table, given = _rows(c)
    if c["op"] == "compact":
        return lens, table, given, max(given, int(given / c["used"])), None
    wishes = _wishes(c, lens)
    return lens, table, given, given + int(_up(wishes[2], c["page"]).sum() * (1 + c["spare"])), wishes


def _numbers(c, seed):
    """The same on the host, with the pages at places of the pool that the seed decides."""
    lens, table, given, n_pages, wishes = _pool(c)
    place = numpy.random.default_rng(seed).permutation(n_pages)
    counts = numpy.empty(n_pages, dtype=numpy.int64)
    counts[place] = _counts(table, lens, c["page"], n_pages, _up(c["prefix"], c["page"]))
    return lens, place[table], counts, place[:_up(c["prefix"], c["page"])], wishes


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = dict(op=c["op"])
    if c["op"] == "prompt":
        lens = _spread(c["batch"], c["len_min"], c["len_max"])
        for name, heads in (("q", c["q_heads"]), ("k", c["kv_heads"]), ("v", c["kv_heads"])):
            shape = (heads, sum(lens), c["head_dim"]) if c["order"] == "hnd" else (sum(lens), heads, c["head_dim"])
            x = torch.empty(shape, dtype=DTYPES[c["dtype"]], device="cuda").normal_(generator=g)
            s[name] = x if c["order"] == "hnd" else x.transpose(0, 1)
        return dict(s, lens=lens, seq_start=_cuda(numpy.cumsum([0] + lens)), causal=c["causal"])
    if c["op"] == "copy":
        r = numpy.random.default_rng(seed)
        for name, order in (("from", c["cache"]), ("to", c["to_cache"])):
            s[name + "_k"], s[name + "_v"] = _cache(g, c, c["pool"], order), _cache(g, c, c["pool"], order)
            s[name + "_pages"] = _cuda(r.permutation(c["pool"])[:c["pages"]])
        return s
    lens, table, counts, prefix, wishes = _numbers(c, seed)
    s.update(k=_cache(g, c, len(counts), c["cache"]), v=_cache(g, c, len(counts), c["cache"]), page=c["page"], table=_cuda(table),
             held=_cuda(lens), counts=_cuda(counts), prefix_pages=_cuda(prefix))
    if c["op"] == "fork":
        parent, keep, room = wishes
        s.update(parent=None if c["mode"] == "step" else _cuda(parent), keep=_cuda(keep), room=_cuda(room), wide=int(_up(room.max(), c["page"])))
    return s


# ------------------------------------------------------------------ the plain forms

def _plain_prompt(s):
    q, k, v = s["q"], s["k"], s["v"]
    H, D = k.shape[0], k.shape[2]
    G = q.shape[0] // H
    o, lse = torch.empty_like(q), torch.empty(q.shape[:2], dtype=torch.float32, device="cuda")
    first = 0
    for n in s["lens"]:
        kf, vf = k[:, first:first + n].float(), v[:, first:first + n].float()
        step = max(1, (1 << 29) // (H * G * n))
        for t in range(0, n, step):
            m = min(step, n - t)
            see = t + m if s["causal"] else n
            at = slice(first + t, first + t + m)
            x = (q[:, at].float() / math.sqrt(D)).reshape(H, G * m, D) @ kf[:, :see].transpose(1, 2)
            x = x.view(H, G, m, see)
            if s["causal"]:
                x.masked_fill_(torch.arange(see, device="cuda") > torch.arange(t, t + m, device="cuda")[:, None], -math.inf)
            top = x.amax(-1, keepdim=True)
            x = x.sub_(top).exp_()
            total = x.sum(-1, keepdim=True)
            r = (x.view(H, G * m, see) @ vf[:, :see]).view(H, G, m, D) / total
            o[:, at] = r.reshape(H * G, m, D).to(o.dtype)
            lse[:, at] = (top + total.log()).view(H * G, m)
        first += n
    return {"o": o, "lse": lse}


def _plain_fork(s):
    table, counts, page = s["table"].long(), s["counts"].long(), s["page"]
    N, (B, W) = counts.numel(), table.shape
    held, keep, room = s["held"].long(), s["keep"].long(), s["room"].long()
    parent = torch.arange(B, device="cuda") if s["parent"] is None else s["parent"].long()
    alive = parent >= 0
    parent = parent.clamp(min=0)
    keep, room = torch.where(alive, keep, 0), torch.where(alive, room, 0)
    room = torch.maximum(room, keep)
    col = torch.arange(W, device="cuda")
    # the last table's rows let go of their pages, the next one's take those that they share
    counts.index_add_(0, table.flatten(), -(col < -(-held // page)[:, None]).long().flatten())
    full, part, total = keep // page, keep % page > 0, -(-room // page)
    old = table[parent]
    counts.index_add_(0, old.flatten(), (col < full[:, None]).long().flatten())
    # a page filled in part stays with the first row that ends in it, if nobody else holds it; the other rows get copies
    last = old.gather(1, full.clamp(max=W - 1)[:, None])[:, 0]
    row = torch.arange(B, device="cuda")
    first = torch.full((N,), B, device="cuda").scatter_reduce_(0, last, torch.where(part, row, B), "amin")
    stays = part & (counts[last] == 0) & (first[last] == row)
    counts.index_add_(0, last, stays.long())
    # the free pages in order, dealt out row by row
    free = counts == 0
    rank = free.cumsum(0) - 1
    pages = torch.full((N + 1,), -1, device="cuda")
    pages[torch.where(free, rank, N)] = torch.arange(N, device="cuda")
    need = total - full - stays.long()
    begin = need.cumsum(0) - need
    counts += free & (rank < need.sum())
    col = torch.arange(s["wide"], device="cuda")
    fresh = pages[(begin[:, None] + col - full[:, None] - stays.long()[:, None]).clamp(0, N - 1)]
    wide = torch.nn.functional.pad(old, (0, max(0, s["wide"] - W)))[:, :s["wide"]]
    out = torch.where(col < full[:, None], wide, torch.where(col < total[:, None], fresh, -1))
    out = torch.where(stays[:, None] & (col == full[:, None]), last[:, None], out)
    # copies: a row that needs none repeats the first one's, or copies a page onto itself where there is none at all
    copies = part & ~stays
    pick = torch.where(copies, row, copies.long().argmax())
    source = last[pick]
    to = torch.where(copies.any(), out.gather(1, full.clamp(max=s["wide"] - 1)[:, None])[:, 0][pick], source)
    kept = (torch.arange(page, device="cuda") < (keep % page)[pick][:, None])[:, None, :, None]
    for x in (s["k"], s["v"]):
        x[to] = torch.where(kept, x[source], x[to])
    return {"table": out.int(), "counts": counts.int(), "k": s["k"], "v": s["v"]}


def _plain_compact(s):
    counts = s["counts"]
    N = counts.numel()
    used = counts > 0
    n = used.sum()
    at = torch.arange(N, device="cuda")
    high, low = used & (at >= n), ~used & (at < n)
    source, to = high.nonzero()[:, 0], low.nonzero()[:, 0]
    place = torch.where(used, at, -1)
    place[source] = to
    for x in (s["k"], s["v"]):
        x[to] = x[source]
    after = torch.zeros_like(counts)
    after[place[used]] = counts[used]
    return {"table": place[s["table"].long()].int(), "prefix_pages": place[s["prefix_pages"].long()].int(), "counts": after, "place": place.int(),
            "used": n.int().view(1), "k": s["k"], "v": s["v"]}


def _plain_copy(s):
    for x in ("k", "v"):
        s["to_" + x][s["to_pages"].long()] = s["from_" + x][s["from_pages"].long()]
    return {"k": s["to_k"], "v": s["to_v"]}


def run(state):
    s = state
    if not own:
        return {"prompt": _plain_prompt, "fork": _plain_fork, "compact": _plain_compact, "copy": _plain_copy}[s["op"]](s)
    from paper_2609_34814_b200 import binding as wb
    if s["op"] == "prompt":
        o, lse = wb.prompt_attn(s["q"], s["k"], s["v"], s["seq_start"], causal=s["causal"], return_lse=True)
        return {"o": o, "lse": lse}
    if s["op"] == "copy":
        wb.cache_copy(wb.PagedCache(s["to_k"], s["to_v"]), s["to_pages"], wb.PagedCache(s["from_k"], s["from_v"]), s["from_pages"])
        return {"k": s["to_k"], "v": s["to_v"]}
    cache = wb.PagedCache(s["k"], s["v"])
    if s["op"] == "fork":
        table, counts = wb.cache_fork(cache, s["table"], s["held"], s["counts"], s["keep"], s["room"], parents=s["parent"], max_pages=s["wide"])
        return {"table": table, "counts": counts, "k": s["k"], "v": s["v"]}
    r = wb.cache_compact(cache, s["counts"], page_table=s["table"], prefix_pages=s["prefix_pages"])
    return {"table": r.page_table, "prefix_pages": r.prefix_pages, "counts": r.page_refs, "place": r.place, "used": r.used, "k": s["k"], "v": s["v"]}


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    c = case
    if c["op"] == "prompt":
        lens = _spread(c["batch"], c["len_min"], c["len_max"])
        pairs = sum(n * (n + 1) // 2 if c["causal"] else n * n for n in lens)
        return {"bytes": sum(lens) * (4 * (c["q_heads"] + c["kv_heads"]) * c["head_dim"] + 4 * c["q_heads"]), "flops": 4 * pairs * c["q_heads"] * c["head_dim"]}
    token = 4 * c["kv_heads"] * c["head_dim"]                              # bytes of a token's keys and values
    if c["op"] == "copy":
        return {"bytes": 2 * c["pages"] * c["page"] * token + 8 * c["pages"], "flops": 0}
    lens, table, given, n_pages, wishes = _pool(c)
    held = int(_up(lens, c["page"]).sum())
    if c["op"] == "fork":
        copied = _next_table(table, lens, _counts(table, lens, c["page"], n_pages, _up(c["prefix"], c["page"])), wishes, c["page"])[2]
        # the last table, the next one, the counts twice, lengths and parents, the copied tokens twice
        return {"bytes": 4 * (held + int(_up(wishes[2], c["page"]).sum()) + 2 * n_pages + 4 * c["batch"]) + 2 * token * sum(n for _, _, n in copied), "flops": 0}
    # counts and tables twice, every page's place, the moved pages twice: of the upper part of a pool as many are in use as its share
    moved = given * (n_pages - given) // n_pages
    return {"bytes": 8 * (held + _up(c["prefix"], c["page"])) + 12 * n_pages + 2 * moved * c["page"] * token, "flops": 0}


# ------------------------------------------------------------------ the definitions

def _next_table(table, lens, counts, wishes, page):
    """(rows as lists of pages, counts, [(from, to, tokens)]) of a fork, row by row."""
    counts = counts.tolist()
    table = [r[:int(n)] for r, n in zip(table.tolist(), _up(lens, page))]
    parent, keep, room = (x.tolist() for x in wishes)
    for r in table:
        for p in r:
            counts[p] -= 1
    rows = []
    for b, n in zip(parent, keep):
        rows.append(table[b][:n // page] if b >= 0 else [])
        for p in rows[-1]:
            counts[p] += 1
    copies = []
    for r, b, n in zip(rows, parent, keep):
        if b >= 0 and n % page:
            last = table[b][n // page]
            if counts[last] == 0:
                counts[last] = 1
                r.append(last)
            else:
                copies.append([last, len(rows), n % page])
                r.append(copies[-1])          # its page follows
    free = iter([p for p, n in enumerate(counts) if n == 0])
    for r, b, n, m in zip(rows, parent, keep, room):
        if r and isinstance(r[-1], list):
            r[-1][1] = next(free)
            r[-1] = r[-1][1]
            counts[r[-1]] = 1
        while b >= 0 and len(r) < _up(max(n, m), page):
            r.append(next(free))
            counts[r[-1]] = 1
    return rows, counts, copies


def _exact_prompt(c, s):
    if work(c)["flops"] > 2e13:
        return None
    H, D = c["kv_heads"], c["head_dim"]
    G = c["q_heads"] // H
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    first = 0
    for n in s["lens"]:
        for h in range(H):
            k, v = s["k"][h, first:first + n].double(), s["v"][h, first:first + n].double()
            for i in range(G * h, G * h + G):
                step = max(1, (1 << 27) // n)
                for t in range(0, n, step):
                    rows = slice(first + t, first + min(t + step, n))
                    x = s["q"][i, rows].double() @ k.t() / math.sqrt(D)
                    if c["causal"]:
                        x = x + torch.full_like(x, -math.inf).triu(t + 1)
                    lse[i, rows] = torch.logsumexp(x, -1)
                    o[i, rows] = torch.softmax(x, -1) @ v
        first += n
    return {"o": o, "lse": lse}


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "prompt":
        return _exact_prompt(c, s)
    if c["op"] == "copy":
        k, v = s["to_k"].double(), s["to_v"].double()
        for a, b in zip(s["from_pages"].tolist(), s["to_pages"].tolist()):
            k[b], v[b] = s["from_k"][a].double(), s["from_v"][a].double()
        return {"k": k, "v": v}
    lens, table, counts, prefix, wishes = _numbers(c, seed)
    k, v = s["k"].double(), s["v"].double()
    if c["op"] == "fork":
        rows, counts, copies = _next_table(table, lens, counts, wishes, c["page"])
        out = numpy.full((len(rows), s["wide"]), -1)
        for b, r in enumerate(rows):
            out[b, :len(r)] = r
        for a, b, n in copies:
            k[b, :, :n], v[b, :, :n] = s["k"][a, :, :n].double(), s["v"][a, :, :n].double()
        return {"table": _cuda(out), "counts": _cuda(counts), "k": k, "v": v}
    used = [p for p, n in enumerate(counts.tolist()) if n > 0]
    spots = iter(sorted(set(range(len(used))) - set(used)))
    place, after = numpy.full(len(counts), -1), numpy.zeros(len(counts), dtype=numpy.int64)
    for p in used:
        place[p] = p if p < len(used) else next(spots)
        after[place[p]] = counts[p]
        if place[p] != p:
            k[place[p]], v[place[p]] = s["k"][p].double(), s["v"][p].double()
    return {"table": _cuda(place[table]), "prefix_pages": _cuda(place[prefix]), "counts": _cuda(after), "place": _cuda(place),
            "used": torch.tensor([len(used)], dtype=torch.int32, device="cuda"), "k": k, "v": v}
