"""Prompts through the calls that serve them, in the order a program makes them, against each sequence by itself in 64 bits: pages given out, prompt
attention, the cache filled, tokens decoded, sequences continued in several ways and ended, the pool compacted, pages moved to another cache."""
import math

import pytest
import torch

from paper_2609_34814_b200 import binding as wb
from paper_2609_34814_b200 import continue_clip as cc
from pages_util import ints, up

pytestmark = pytest.mark.gpu


class Program:
    """A program that serves prompts.  It holds a pool of pages, a table, counts; and, for the test, what every sequence's keys and values are."""

    def __init__(self, heads, kv_heads, dim, page, pages, dtype, seed):
        self.heads, self.kv_heads, self.dim, self.page, self.dtype = heads, kv_heads, dim, page, dtype
        self.cache = wb.PagedCache(*(torch.full((pages, kv_heads, page, dim), math.nan, dtype=dtype, device="cuda") for _ in range(2)))
        self.refs, self.table, self.held = torch.zeros(pages, dtype=torch.int32, device="cuda"), ints([]).view(0, 0), []
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.k, self.v = [], []
        self.status = ints([0] * 4)

    def draw(self, tokens):
        return [torch.randn((tokens, h, self.dim), generator=self.g, device="cuda").to(self.dtype).transpose(0, 1) for h in (self.heads, self.kv_heads, self.kv_heads)]

    def fork(self, parents, keep, room):
        self.table, self.refs = wb.cache_fork(self.cache, self.table, ints(self.held), self.refs, ints(keep), ints(room), parents=ints(parents),
                                              max_pages=max([up(n, self.page) for n in room] + [1]), dev_status=self.status)
        none = torch.zeros((self.kv_heads, 0, self.dim), dtype=self.dtype, device="cuda")
        of = lambda x: [x[p][:, :n] if p >= 0 and x else none for p, n in zip(parents, keep)]  # noqa: E731
        self.k, self.v, self.held = of(self.k), of(self.v), list(room)

    def append(self, k, v, new):
        start = ints([0] + torch.tensor(new).cumsum(0).tolist())
        at = 0
        for b, n in enumerate(new):
            self.k[b], self.v[b] = (torch.cat([x[b], y[:, at:at + n]], 1) for x, y in ((self.k, k), (self.v, v)))
            at += n
        wb.cache_append(self.cache, k, v, start, ints([x.shape[1] for x in self.k]), self.table, dev_status=self.status)
        return start

    def expected(self, q, new):
        out, at = [], 0
        for b, n in enumerate(new):
            k, v = (x[b].double().repeat_interleave(self.heads // self.kv_heads, 0) for x in (self.k, self.v))
            x = q[:, at:at + n].double() @ k.transpose(1, 2) / math.sqrt(self.dim)
            have = k.shape[1]
            x = x.masked_fill(torch.arange(have, device="cuda") > torch.arange(have - n, have, device="cuda")[:, None], -math.inf)
            w = torch.softmax(x, -1)
            # p and the result in the tensors' type: half a step each, and fp32 sums
            out.append((w @ v, (w @ v.abs()) * 1.5 * torch.finfo(self.dtype).eps / 2 + (w @ v).abs() * torch.finfo(self.dtype).eps / 2 + 1e-6))
            at += n
        return (torch.cat(x, 1) for x in zip(*out))

    def check(self, o, q, new):
        want, tol = self.expected(q, new)
        assert ((o.double() - want).abs() <= tol).all()

    def decode(self):
        """one token of every sequence"""
        B = len(self.held)
        have = [x.shape[1] for x in self.k]
        self.fork(list(range(B)), have, [n + 1 for n in have])
        q, k, v = self.draw(B)
        start = self.append(k, v, [1] * B)
        o = wb.prefix_attn(self.cache, q, start, ints([n + 1 for n in have]), self.table, dev_status=self.status)
        self.check(o, q, [1] * B)


@pytest.mark.parametrize("heads, kv_heads, dim, page, dtype", [(8, 2, 128, 16, torch.bfloat16), (6, 2, 64, 64, torch.float16)])
def test_prompts_decoded_forked_compacted(heads, kv_heads, dim, page, dtype):
    p = Program(heads, kv_heads, dim, page, 300, dtype, seed=dim)
    lens = [70, 1, 333, 16, 129]
    # the prompts: pages, attention, cache
    p.fork([-1] * 5, [0] * 5, [0] * 5)
    assert not p.refs.any() and (p.table == -1).all()
    table = ints([[-1] * 0] * 5)
    p.table, p.held = table, [0] * 5
    p.fork([0, 1, 2, 3, 4], [0] * 5, lens)
    assert int(p.refs.sum()) == sum(up(n, page) for n in lens)
    q, k, v = p.draw(sum(lens))
    start = p.append(k, v, lens)
    o, lse = wb.prompt_attn(q, k, v, start, return_lse=True, dev_status=p.status)
    p.check(o, q, lens)
    # the same from the cache
    o2, lse2 = wb.prefix_attn(p.cache, q, start, ints(lens), p.table, return_lse=True, dev_status=p.status)
    eps = torch.finfo(dtype).eps
    assert ((o.double() - o2.double()).abs() <= 2 * eps * (o.double().abs() + 4)).all() and ((lse - lse2).abs() <= 1e-4).all()
    for _ in range(3):
        p.decode()
    # the first goes on in three ways, the third in two of which one is cut back, the second ends
    have = [x.shape[1] for x in p.k]
    p.fork([0, 2, 0, 3, 4, 0, 2], [have[0], have[2], have[0], have[3], have[4], have[0], 200], [have[0] + 5] * 1 + [have[2], have[0], have[3], have[4], have[0] + 40, 201])
    for _ in range(2):
        p.decode()
    # the pool to its front, then on
    before = int((p.refs > 0).sum())
    r = wb.cache_compact(p.cache, p.refs, page_table=p.table)
    p.table, p.refs = r.page_table, r.page_refs
    assert r.used.item() == before == int((p.refs > 0).sum()) and not p.refs[before:].any()
    p.cache.k[before:] = math.nan
    p.cache.v[before:] = math.nan
    for _ in range(2):
        p.decode()
    # two sequences move to another program's cache, whose pages hold their tokens token by token
    small = [torch.full((60, page, kv_heads, dim), math.nan, dtype=dtype, device="cuda").transpose(1, 2) for _ in range(2)]
    pages = [p.table[b, :up(p.held[b], page)] for b in (1, 4)]
    count = [x.numel() for x in pages]
    to = torch.randperm(60, device="cuda")[:sum(count)].int()
    wb.cache_copy(wb.PagedCache(*small), to, p.cache, torch.cat(pages), dev_status=p.status)
    other = Program(heads, kv_heads, dim, page, 60, dtype, seed=5)
    other.cache = wb.PagedCache(*small)
    other.table = torch.full((2, max(count)), -1, dtype=torch.int32, device="cuda")
    other.table[0, :count[0]], other.table[1, :count[1]] = to[:count[0]], to[count[0]:]
    other.refs[to.long()] = 1
    other.held, other.k, other.v = [p.held[1], p.held[4]], [p.k[1], p.k[4]], [p.v[1], p.v[4]]
    other.decode()
    # everything ends
    p.fork([-1], [0], [0])
    assert not p.refs.any() and p.status.tolist() == other.status.tolist() == [0] * 4


def test_chosen_continuations_go_on():
    """A clip whose continuations are chosen between frames gives what the chosen ones alone would give."""
    heads, dim, grid, frames, new_frames = 2, 64, (5, 9), 3, 3
    layers = [cc.ClipLayer(heads, dim, grid, frames, new_frames, 4, page=16) for _ in range(2)]
    g = torch.Generator(device="cuda").manual_seed(1)
    draw = lambda n: [torch.randn((heads, n, dim), generator=g, device="cuda").bfloat16() for _ in range(3)]  # noqa: E731
    clip = draw(layers[0].clip)
    for layer in layers:
        layer.start(*clip, cc.band_mask(heads, -(-layer.clip // 64), 1))
    n = layers[0].frame
    x = draw(4 * n)
    parents = [2, 2, 0, 2]
    first = [layers[0].step(*x), layers[1].step(*(torch.cat([t[:, p * n:(p + 1) * n] for p in parents], 1) for t in x))]
    for b, p in enumerate(parents):
        assert torch.equal(first[1][:, b * n:(b + 1) * n], first[0][:, p * n:(p + 1) * n])
    layers[0].choose(parents)
    y = draw(4 * n)
    assert torch.equal(layers[0].step(*y), layers[1].step(*y))
    layers[0].choose([3, 1])
    z = draw(2 * n)
    o = layers[0].step(*z)
    layers[1].choose(torch.tensor([3, 1]))
    assert torch.equal(o, layers[1].step(*z))
    assert layers[0].status.tolist() == layers[1].status.tolist() == [0] * 4
    with pytest.raises(ValueError):
        layers[0].choose([0, 1, 0])


def test_command_chooses(capsys):
    cc.main(["--heads", "2", "--frames", "2", "--height", "6", "--width", "10", "--continuations", "3", "--new-frames", "3", "--choose"])
    out = capsys.readouterr().out
    assert out.count("go on") == 2 and "frame 2: 3 continuations" in out
