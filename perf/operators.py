"""Rotary positions, the paged key/value cache and attention over a shared prefix, as measurable cases.

A program that continues one clip (or one prompt) in several ways keeps the keys and values of the common
past once, in a paged cache, and each continuation's own behind it.  Per layer and step it calls

  rope    queries and keys are rotated by their positions: one axis for a token sequence, three (frame, height,
          width) for video; half or interleaved pairs, all or part of the head, frequencies scaled for contexts
          longer than the trained one.  The gradient is the rotation backwards.
  append  the step's new keys (rotated on the way) and values go to their pages, the queries are rotated beside them.
  attend  every query attends to the shared prefix and to its own continuation: one new token a sequence,
          some (drafts), or the whole token grid of a video frame.

Frequencies are a table of phase steps, one a pair: turns per position, in units of 2^-64 turns.  A position
times a step, cut to 64 bits, is the angle's fraction of a turn with no rounding that grows with the position.

Tensors are [heads, tokens, head_dim] views (any strides); the new tokens of all sequences lie one after another,
`seq_start` says where each begins.  `kv_len` counts a sequence's own keys once its new ones are in.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}

ROPE = dict(op="rope", tokens=8, q_heads=32, k_heads=8, head_dim=128, rot_dim=128, dtype="bf16", interleaved=False, axes=1,
            grid_h=30, grid_w=52, base=10000.0, scaling="none", factor=1.0, trained=8192, start=0, grad=False, order="nhd")
CACHE = dict(batch=8, new_min=1, new_max=1, own_min=1, own_max=256, prefix=0, q_heads=32, kv_heads=8, head_dim=128, page=16,
             dtype="bf16", cache="hnd")
APPEND = dict(CACHE, op="append", rot_dim=128, interleaved=False, axes=1, grid_h=30, grid_w=52, base=10000.0, scaling="none", factor=1.0,
              trained=8192)
ATTEND = dict(CACHE, op="attend", causal=True)


def listed():
    return [
        # eight sequences decode one token each far beyond the trained length: launch and latency
        dict(ROPE, name="rope_tokens", base=500000.0, scaling="parts", factor=16.0, start=100000),
        # a whole 480p clip (21 latent frames of 30 x 52 tokens), 40 heads, in front of the block-sparse attention
        dict(ROPE, name="rope_clip", tokens=32760, q_heads=40, k_heads=40, interleaved=True, axes=3, order="hnd"),
        # a training step's gradients in 32 bits: an odd number of tokens, 40 of 96 channels rotated
        dict(ROPE, name="rope_grad_part", tokens=4099, q_heads=12, k_heads=4, head_dim=96, rot_dim=40, dtype="fp32", scaling="linear",
             factor=4.0, start=20000, grad=True),
        # one decoded token of sixteen continuations into 16-token pages
        dict(APPEND, name="append_tokens", batch=16, own_max=1000, prefix=8192, base=500000.0),
        # four continuations add a video frame each
        dict(APPEND, name="append_frames", batch=4, new_min=1560, new_max=1560, own_min=1560, own_max=6240, prefix=32760, q_heads=40,
             kv_heads=40, page=128, interleaved=True, axes=3),
        # prompts of 1 to 700 tokens, fp16, part of a head of 64, token-major pages
        dict(APPEND, name="append_ragged", batch=23, new_min=1, new_max=700, own_min=1, own_max=2500, prefix=1000, q_heads=28, kv_heads=4,
             head_dim=64, page=32, dtype="fp16", cache="nhd", rot_dim=32, scaling="ntk", factor=8.0),
        # the smallest: three continuations of a short prompt, one token each
        dict(ATTEND, name="attend_few", batch=3, own_max=40, prefix=500, q_heads=8, kv_heads=2, head_dim=64),
        # ordinary decoding: 32 continuations of different lengths
        dict(ATTEND, name="attend_tokens", batch=32, own_max=2000, prefix=8192),
        # a very long common context, 64 continuations: as much arithmetic as memory traffic
        dict(ATTEND, name="attend_long", batch=64, own_max=1000, prefix=131072, page=64),
        # as many key heads as query heads behind a 480p clip, one token each
        dict(ATTEND, name="attend_clip_tokens", batch=16, own_max=1560, prefix=32760, q_heads=40, kv_heads=40, page=64),
        # the next frame of four continuations on one of eight GPUs (5 of 40 heads): the largest
        dict(ATTEND, name="attend_frames", batch=4, new_min=1560, new_max=1560, own_min=1560, own_max=4680, prefix=32760, q_heads=5,
             kv_heads=5, page=128, causal=False),
        # drafts and short prompts: 1 to 70 new tokens, fp16, head_dim 64, seven query heads a key head, token-major pages
        dict(ATTEND, name="attend_drafts", batch=13, new_min=1, new_max=70, own_min=1, own_max=900, prefix=3001, q_heads=28, kv_heads=4,
             head_dim=64, page=128, dtype="fp16", cache="nhd"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng):
    kv = rng.choice([1, 2, 4, 5, 8, 10, 40])
    return kv * rng.choice([1, 1, 2, 3, 4, 5, 7, 8]) if kv < 40 else 40, kv


def _positions_of(rng, rot_max):
    axes = rng.choice([1, 1, 3])
    rot = rng.choice([rot_max, rot_max, rot_max // 2, rot_max // 4])
    scaling = rng.choice(["none", "linear", "ntk", "parts"])
    return dict(axes=axes, rot_dim=max(rot, 16), interleaved=rng.random() < 0.5, scaling=scaling,
                factor=1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0, 16.0]), base=rng.choice([10000.0, 500000.0]))


def draw(rng):
    """One more case: any operator, length, head layout, page, type and rotation of the ranges above."""
    op = rng.choice(["rope", "append", "attend", "attend"])
    q_heads, kv_heads = _heads(rng)
    if op == "rope":
        head_dim = rng.choice([64, 80, 96, 128, 128, 256])
        case = dict(ROPE, q_heads=q_heads, k_heads=rng.choice([0, kv_heads]), head_dim=head_dim, dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]),
                    grad=rng.random() < 0.4, order=rng.choice(["hnd", "nhd"]), start=_log(rng, 1, 1000000), **_positions_of(rng, head_dim))
        most = 32760 * 80 * 128 // ((q_heads + case["k_heads"]) * head_dim)
        return dict(case, tokens=_log(rng, 1, min(most, 200000)))
    case = dict(batch=_log(rng, 1, 200), q_heads=q_heads, kv_heads=kv_heads, head_dim=rng.choice([64, 128, 128]), page=rng.choice([16, 16, 32, 64, 128, 256]),
                dtype=rng.choice(["bf16", "bf16", "fp16"]), cache=rng.choice(["hnd", "nhd"]))
    new = rng.choice([1, 1, 1, _log(rng, 2, 100), _log(rng, 2, 1560)])
    new = max(1, min(new, 8000 // case["batch"]))
    case.update(new_min=new if rng.random() < 0.5 else 1, new_max=new, own_max=new + _log(rng, 1, 3000))
    case["own_min"] = rng.choice([1, new])
    token = case["kv_heads"] * case["head_dim"] * 4                       # bytes of one cached token
    case["own_max"] = max(new, min(case["own_max"], (1 << 30) // (token * case["batch"])))
    case["own_min"] = min(case["own_min"], case["own_max"])
    if op == "append":
        return dict(APPEND, **case, prefix=_log(rng, 1, 200000), **_positions_of(rng, case["head_dim"]))
    rows = case["batch"] * new * q_heads
    prefix = 0 if rng.random() < 0.1 else _log(rng, 1, min(140000, (1 << 29) // rows, (1 << 30) // token))
    # (scores of the own part in the plain form: batch x new x q_heads x own_max numbers)
    case["own_max"] = max(new, min(case["own_max"], (1 << 29) // rows))
    case["own_min"] = min(case["own_min"], case["own_max"])
    return dict(ATTEND, **case, prefix=prefix, causal=rng.random() < 0.7)


# ------------------------------------------------------------------ what a program has in hand

def _spread(n, lo, hi, step):
    """n whole numbers from lo to hi, unlike their neighbours, both ends among them."""
    return [hi if b == 0 else lo if b == n - 1 else lo + int((b * step) % 1.0 * (hi - lo + 1)) for b in range(n)]


def _lengths(c):
    """(new tokens, own keys with the new ones in) of every sequence."""
    new = _spread(c["batch"], c["new_min"], c["new_max"], 0.7548776662466927)
    kept = _spread(c["batch"], c["own_min"], c["own_max"], 0.6180339887498949)
    return new, [max(n, k) for n, k in zip(new, kept)]


def _axis_pairs(c):
    """Pairs of each axis: all, or 22 : 21 : 21 of every 64 for frame, height and width."""
    pairs = c["rot_dim"] // 2
    return [pairs] if c["axes"] == 1 else [pairs - 2 * (pairs // 3), pairs // 3, pairs // 3]


def _angles(c):
    """(radians a position for every pair, factor on the rotated channels)"""
    theta, amplitude, s = [], 1.0, c["factor"]
    for pairs in _axis_pairs(c):
        base = c["base"] * s ** (2 * pairs / (2 * pairs - 2)) if c["scaling"] == "ntk" and pairs > 1 else c["base"]
        for i in range(pairs):
            t = base ** (-i / pairs)
            if c["scaling"] == "linear":
                t /= s
            elif c["scaling"] == "parts":
                # pairs that turn over 32 times in the trained length stay, those that turn less than once are stretched
                keep = min(1.0, max(0.0, (c["trained"] * t / (2 * math.pi) - 1.0) / 31.0))
                t = t * keep + t / s * (1.0 - keep)
            theta.append(t)
    if c["scaling"] == "parts":
        amplitude = 0.1 * math.log(s) + 1.0
    return theta, amplitude


def _rotation(c, device):
    theta, amplitude = _angles(c)
    steps = torch.tensor([int(t / (2 * math.pi) * 2.0 ** 64) for t in theta], dtype=torch.int64, device=device)
    return dict(steps=steps, axis_pairs=_axis_pairs(c), amplitude=amplitude, interleaved=c["interleaved"], rot_dim=c["rot_dim"])


def _grid(c, first, count):
    """Positions of tokens first .. first + count - 1: themselves, or frame, height and width on the video's grid."""
    t = first + torch.arange(count, dtype=torch.int64)
    if c["axes"] == 1:
        return t[None]
    per = c["grid_h"] * c["grid_w"]
    return torch.stack([t // per, t % per // c["grid_w"], t % c["grid_w"]])


def _normal(g, shape, dtype, order="hnd"):
    """[heads, tokens, head_dim], the tokens outermost in memory for "nhd"."""
    if order == "nhd":
        shape = (shape[1], shape[0], shape[2])
    x = torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=g)
    return x.transpose(0, 1) if order == "nhd" else x


def _cache(g, c, pages, dtype):
    """[pages, heads, page, head_dim], the page's tokens outermost in memory for "nhd"."""
    H, P, D = c["kv_heads"], c["page"], c["head_dim"]
    shape = (pages, P, H, D) if c["cache"] == "nhd" else (pages, H, P, D)
    x = torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=g)
    return x.transpose(1, 2) if c["cache"] == "nhd" else x


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dtype = DTYPES[c["dtype"]]
    s = dict(op=c["op"])
    if c["op"] == "rope":
        s["q"] = _normal(g, (c["q_heads"], c["tokens"], c["head_dim"]), dtype, c["order"])
        s["k"] = _normal(g, (c["k_heads"], c["tokens"], c["head_dim"]), dtype, c["order"]) if c["k_heads"] else None
        s["positions"] = _grid(c, c["start"], c["tokens"]).to(torch.int32).cuda()
        s["grad"] = c["grad"]
        return dict(s, **_rotation(c, "cuda"))

    new, kept = _lengths(c)
    shared = -(-c["prefix"] // c["page"])
    wide = -(-max(kept) // c["page"])
    owned = [-(-n // c["page"]) for n in kept]
    order = torch.randperm(shared + sum(owned), generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    table = torch.zeros((c["batch"], wide), dtype=torch.int32)
    at = shared
    for b, n in enumerate(owned):
        table[b, :n] = order[at:at + n]
        at += n
    s.update(seq_start=torch.tensor([0] + new).cumsum(0).to(torch.int32).cuda(), kv_len=torch.tensor(kept, dtype=torch.int32).cuda(),
             page_table=table.cuda(), prefix=c["prefix"], prefix_pages=order[:shared].cuda(), longest=max(new))
    pages = shared + sum(owned) if c["op"] == "attend" else int(order.max()) + 1
    s["k_cache"], s["v_cache"] = _cache(g, c, pages, dtype), _cache(g, c, pages, dtype)
    # queries and keys as they come out of a projection: token by token
    s["q"] = _normal(g, (c["q_heads"], sum(new), c["head_dim"]), dtype, "nhd")
    if c["op"] == "attend":
        return dict(s, causal=c["causal"])
    s["k"] = _normal(g, (c["kv_heads"], sum(new), c["head_dim"]), dtype, "nhd")
    s["v"] = _normal(g, (c["kv_heads"], sum(new), c["head_dim"]), dtype, "nhd")
    if c["axes"] > 1:       # a program with a grid says where its tokens are; a token sequence is counted through
        s["positions"] = torch.cat([_grid(c, c["prefix"] + k - n, n) for n, k in zip(new, kept)], 1).to(torch.int32).cuda()
    else:
        s["positions"] = None
    return dict(s, **_rotation(c, "cuda"))


# ------------------------------------------------------------------ the plain forms

def _cos_sin(s, positions):
    """[tokens, pairs] each, from whole fractions of a turn."""
    axis = torch.repeat_interleave(torch.arange(len(s["axis_pairs"]), device="cuda"), torch.tensor(s["axis_pairs"], device="cuda"),
                                   output_size=s["rot_dim"] // 2)
    turns = (positions.long()[axis].t() * s["steps"]) >> 32
    angle = turns.float() * (2 * math.pi / 2.0 ** 32)
    return angle.cos() * s["amplitude"], angle.sin() * s["amplitude"]


def _rotate(x, cos, sin, rot, interleaved):
    f = x.float()
    a, b = (f[..., 0:rot:2], f[..., 1:rot:2]) if interleaved else (f[..., :rot // 2], f[..., rot // 2:rot])
    u, w = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([u, w], -1).flatten(-2) if interleaved else torch.cat([u, w], -1)
    return torch.cat([turned, f[..., rot:]], -1).to(x.dtype)


def _plain_rope(s):
    cos, sin = _cos_sin(s, s["positions"])
    if s["grad"]:
        sin = -sin
    q = _rotate(s["q"], cos, sin, s["rot_dim"], s["interleaved"])
    return {"q": q} if s["k"] is None else {"q": q, "k": _rotate(s["k"], cos, sin, s["rot_dim"], s["interleaved"])}


def _places(s):
    """Of every new token: its sequence, its number among the new ones, its place among the sequence's own keys."""
    new = s["seq_start"].diff().long()
    b = torch.repeat_interleave(torch.arange(new.numel(), device="cuda"), new, output_size=s["q"].shape[1])
    i = torch.arange(b.numel(), device="cuda") - s["seq_start"].long()[b]
    return b, i, s["kv_len"].long()[b] - new[b] + i


def _plain_append(s):
    page = s["k_cache"].shape[2]
    b, _, place = _places(s)
    cos, sin = _cos_sin(s, (s["prefix"] + place)[None] if s["positions"] is None else s["positions"])
    to = s["page_table"][b, place // page].long()
    s["k_cache"][to, :, place % page] = _rotate(s["k"], cos, sin, s["rot_dim"], s["interleaved"]).transpose(0, 1)
    s["v_cache"][to, :, place % page] = s["v"].transpose(0, 1)
    return {"q": _rotate(s["q"], cos, sin, s["rot_dim"], s["interleaved"]), "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _plain_attend(s):
    q, k, v = s["q"], s["k_cache"], s["v_cache"]
    T, D, H, B = q.shape[1], q.shape[2], k.shape[1], s["kv_len"].numel()
    G, P, N, M = q.shape[0] // H, s["prefix"], s["longest"], s["page_table"].shape[1] * k.shape[2]
    qf = q.float().view(H, G, T, D).transpose(1, 2) / math.sqrt(D)                              # [H, T, G, D]
    # the prefix, for all queries at once
    kp, vp = (x[s["prefix_pages"].long()].transpose(0, 1).reshape(H, -1, D)[:, :P].float() for x in (k, v))
    sp = qf.reshape(H, T * G, D) @ kp.transpose(1, 2)                                           # [H, T * G, P]
    top = torch.cat([sp, sp.new_full((H, T * G, 1), -math.inf)], -1).amax(-1).view(H, T, G)
    # each sequence's own keys, its queries padded to the longest
    ko, vo = (x[s["page_table"].long()].permute(2, 0, 1, 3, 4).reshape(H, B, M, D).float() for x in (k, v))
    b, i, place = _places(s)
    padded = (s["seq_start"][:-1, None].long() + torch.arange(N, device="cuda")).clamp(max=T - 1)  # [B, N]
    so = qf[:, padded].reshape(H, B, N * G, D) @ ko.transpose(2, 3)                             # [H, B, N * G, M]
    sees = torch.zeros((B, N), dtype=torch.int64, device="cuda")
    sees[b, i] = place + 1 if s["causal"] else s["kv_len"].long()[b]
    hidden = torch.arange(M, device="cuda") >= sees[..., None]                                  # [B, N, M]
    so = so.view(H, B, N, G, M).masked_fill_(hidden[:, :, None], -math.inf)
    top = torch.maximum(top, so.amax(-1)[:, b, i])                                              # [H, T, G]
    sp = sp.sub_(top.view(H, T * G, 1)).exp_()
    so = so.sub_(top[:, padded][..., None]).masked_fill_(hidden[:, :, None], -math.inf).exp_()
    total = sp.sum(-1).view(H, T, G) + so.sum(-1)[:, b, i]
    out = (sp @ vp).view(H, T, G, D) + (so.view(H, B, N * G, M) @ vo).view(H, B, N, G, D)[:, b, i]
    o = (out / total[..., None]).transpose(1, 2).reshape(H * G, T, D).to(q.dtype)
    return {"o": o, "lse": (top + total.log()).transpose(1, 2).reshape(H * G, T)}


def run(state):
    s = state
    if not own:
        return {"rope": _plain_rope, "append": _plain_append, "attend": _plain_attend}[s["op"]](s)
    from paper_2609_34814_b200 import binding as wb
    if s["op"] == "rope":
        q, k = wb.rope(s["q"], s["positions"], s["steps"], k=s["k"], interleaved=s["interleaved"], axis_pairs=s["axis_pairs"],
                       amplitude=s["amplitude"], inverse=s["grad"])
        return {"q": q} if k is None else {"q": q, "k": k}
    cache = wb.PagedCache(s["k_cache"], s["v_cache"])
    if s["op"] == "append":
        q = wb.cache_append(cache, s["k"], s["v"], s["seq_start"], s["kv_len"], s["page_table"], positions=s["positions"], freqs=s["steps"],
                            q=s["q"], prefix_len=s["prefix"], interleaved=s["interleaved"], axis_pairs=s["axis_pairs"], amplitude=s["amplitude"])
        return {"q": q, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    o, lse = wb.prefix_attn(cache, s["q"], s["seq_start"], s["kv_len"], s["page_table"], s["prefix_pages"], s["prefix"], causal=s["causal"],
                            return_lse=True)
    return {"o": o, "lse": lse}


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    c = case
    size = 4 if c["dtype"] == "fp32" else 2
    if c["op"] == "rope":
        numbers = c["tokens"] * (c["q_heads"] + c["k_heads"]) * c["head_dim"]
        pairs = c["tokens"] * (c["q_heads"] + c["k_heads"]) * c["rot_dim"] // 2
        return {"bytes": 2 * size * numbers + 4 * c["axes"] * c["tokens"] + 4 * c["rot_dim"], "flops": 6 * pairs}
    new, kept = _lengths(c)
    T, D = sum(new), c["head_dim"]
    if c["op"] == "append":
        numbers = T * (c["q_heads"] + 2 * c["kv_heads"]) * D
        return {"bytes": 2 * size * numbers + 12 * T, "flops": 6 * T * (c["q_heads"] + c["kv_heads"]) * c["rot_dim"] // 2}
    seen = sum(n * c["prefix"] + (n * k - n * (n - 1) // 2 if c["causal"] else n * k) for n, k in zip(new, kept))
    return {"bytes": 2 * size * T * c["q_heads"] * D + 4 * T * c["q_heads"] + 2 * size * (c["prefix"] + sum(kept)) * c["kv_heads"] * D,
            "flops": 4 * seen * c["q_heads"] * D}


# ------------------------------------------------------------------ the definitions, in 64 bits

def _turn64(x, positions, theta, axis_pairs, amplitude, rot, interleaved, sign):
    """Pairs as complex numbers times amplitude * e^(i angle)."""
    x = x.double()
    first = 0
    angle = []
    for a, n in enumerate(axis_pairs):
        angle.append(positions[a].double()[:, None] * torch.tensor(theta[first:first + n], dtype=torch.float64, device="cuda"))
        first += n
    angle = torch.cat(angle, 1)
    turn = torch.polar(torch.full_like(angle, amplitude), sign * angle)
    head = x[..., :rot]
    pairs = head.unflatten(-1, (rot // 2, 2)) if interleaved else head.unflatten(-1, (2, rot // 2)).transpose(-1, -2)
    turned = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
    x[..., :rot] = (turned if interleaved else turned.transpose(-1, -2)).flatten(-2)
    return x


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] != "attend":
        theta, amplitude = _angles(c)
        if c["op"] == "rope":
            turn = lambda x: _turn64(x, s["positions"], theta, s["axis_pairs"], amplitude, c["rot_dim"], c["interleaved"], -1 if c["grad"] else 1)  # noqa: E731
            return {"q": turn(s["q"])} if s["k"] is None else {"q": turn(s["q"]), "k": turn(s["k"])}
    new, kept = _lengths(c)
    page = c["page"]
    if c["op"] == "append":
        positions = s["positions"]
        if positions is None:
            positions = torch.cat([torch.arange(c["prefix"] + k - n, c["prefix"] + k) for n, k in zip(new, kept)])[None].cuda()
        q, k = (_turn64(x, positions, theta, s["axis_pairs"], amplitude, c["rot_dim"], c["interleaved"], 1) for x in (s["q"], s["k"]))
        kc, vc, table, t = s["k_cache"].double(), s["v_cache"].double(), s["page_table"].long().cpu(), 0
        for b, (n, have) in enumerate(zip(new, kept)):
            place = torch.arange(have - n, have)
            to = table[b, place // page].cuda()
            kc[to, :, (place % page).cuda()] = k[:, t:t + n].transpose(0, 1)
            vc[to, :, (place % page).cuda()] = s["v"][:, t:t + n].double().transpose(0, 1)
            t += n
        return {"q": q, "k_cache": kc, "v_cache": vc}
    if work(c)["flops"] > 2e12:
        return None
    H, D, P = c["kv_heads"], c["head_dim"], c["prefix"]
    G, T = c["q_heads"] // H, sum(new)
    o = torch.zeros((H * G, T, D), dtype=torch.float64, device="cuda")
    lse = torch.full((H * G, T), -math.inf, dtype=torch.float64, device="cuda")
    table = s["page_table"].long()

    def sums(q, k, v, ends):
        """log of the sum of exponentials, and the mean of v by them; a query sees the keys before its end"""
        x = q @ k.t() / math.sqrt(D)
        if ends is not None:
            x = x.masked_fill(torch.arange(k.shape[0], device="cuda") >= ends[:, None], -math.inf)
        return torch.logsumexp(x, -1), torch.softmax(x, -1) @ v

    for h in range(H):
        kh, vh = s["k_cache"][:, h], s["v_cache"][:, h]
        q = s["q"][h * G:(h + 1) * G].double()
        parts = []
        if P:
            kp, vp = (x[s["prefix_pages"].long()].reshape(-1, D)[:P].double() for x in (kh, vh))
            step = max(1, (1 << 27) // (G * P))
            for t in range(0, T, step):
                n = min(step, T - t)
                parts.append((t, n) + sums(q[:, t:t + n].reshape(G * n, D), kp, vp, None))
        t = 0
        for b, (n, have) in enumerate(zip(new, kept)):
            ko, vo = (x[table[b, :-(-have // page)]].reshape(-1, D)[:have].double() for x in (kh, vh))
            ends = (torch.arange(have - n, have, device="cuda") + 1 if c["causal"] else torch.full((n,), have, device="cuda")).repeat(G)
            parts.append((t, n) + sums(q[:, t:t + n].reshape(G * n, D), ko, vo, ends))
            t += n
        for t, n, part, mean in parts:
            part, mean, rows = part.view(G, n), mean.view(G, n, D), slice(h * G, (h + 1) * G)
            both = torch.logaddexp(lse[rows, t:t + n], part)
            o[rows, t:t + n] = o[rows, t:t + n] * (lse[rows, t:t + n] - both).exp()[..., None] + mean * (part - both).exp()[..., None]
            lse[rows, t:t + n] = both
    return {"o": o, "lse": lse}
