"""Rotary positions and appending to the paged cache, against the definition in 64 bits."""
import math

import pytest
import torch

from paper_2609_34814_b200 import binding as wb
from tests.serving_util import rotated, rotation_tolerance

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def radians(freqs):
    return freqs.cpu().double() / 2.0 ** 64 * (2 * math.pi)


def close(got, want, x, rot, interleaved, amplitude, dtype):
    tol, unit = rotation_tolerance(x, rot, interleaved, amplitude, dtype)
    off = (got.double().cpu() - want).abs()
    bound = tol + unit * want.abs() + (2.0 ** -25 if dtype == torch.float16 else 0.0)
    assert bool((off <= bound).all()), float((off - bound).max())


def axes_of(pairs, axes):
    return [pairs] if axes == 1 else [pairs - 2 * (pairs // 3), pairs // 3, pairs // 3]


CASES = [
    # tokens, q heads, k heads, dim, rot, type, interleaved, axes, first position, token-major
    (1, 1, 0, 2, 2, "fp32", False, 1, 7, True),
    (1, 32, 8, 128, 128, "bf16", False, 1, 131071, True),
    (3, 5, 1, 128, 128, "bf16", True, 3, 0, False),
    (33, 4, 4, 96, 40, "fp32", False, 1, 1000000, True),
    (33, 4, 2, 96, 40, "bf16", True, 1, 1000, False),
    (257, 3, 1, 64, 32, "fp16", False, 1, 5, True),
    (19, 2, 2, 80, 20, "bf16", False, 1, 100, False),       # rot_dim/2 = 10: no wide vectors
    (19, 2, 2, 80, 20, "fp16", True, 3, 100, False),
    (5, 7, 3, 33, 6, "fp32", True, 1, 2000000000, True),    # odd head_dim
    (4, 2, 1, 512, 512, "bf16", False, 1, 9, True),
    (4, 2, 1, 511, 2, "fp32", True, 1, 9, True),
    (1000, 40, 40, 128, 128, "bf16", True, 3, 0, False),
    (130, 1, 0, 256, 64, "fp32", False, 2, -50, False),     # positions below zero
]


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES, ids=[f"{c[0]}x{c[1]}+{c[2]}x{c[3]}r{c[4]}{c[5]}{'i' if c[6] else 'h'}{c[7]}" for c in CASES])
@pytest.mark.parametrize("inverse", [False, True])
def test_rope_matches_definition(case, inverse):
    tokens, qh, kh, dim, rot, kind, inter, axes, first, token_major = case
    dtype = TYPES[kind]
    g = torch.Generator().manual_seed(tokens + dim)
    q, k = ((torch.randn((h, tokens, dim), generator=g) * 3).to(dtype) for h in (qh, max(kh, 1)))
    pairs = rot // 2
    split = [pairs, 0] if axes == 2 and pairs < 2 else [pairs - pairs // 2, pairs // 2] if axes == 2 else axes_of(pairs, axes)
    freqs, _ = wb.rope_freqs(rot, device="cpu")
    positions = torch.stack([first + (a + 1) * torch.arange(tokens) for a in range(axes)]).clamp(max=2 ** 31 - 1).to(torch.int32)
    amplitude = 1.25
    lay = (lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)) if token_major else (lambda t: t)
    qo, ko = wb.rope(lay(q.cuda()), positions.cuda(), freqs.cuda(), k=lay(k.cuda()) if kh else None, interleaved=inter, axis_pairs=split,
                     amplitude=amplitude, inverse=inverse)
    for x, got in ((q, qo), (k, ko)):
        if got is None:
            assert not kh
            continue
        want = rotated(x.double(), positions, radians(freqs), split, inter, amplitude, inverse)
        close(got, want, x.double(), rot, inter, amplitude, dtype)
        assert torch.equal(got[..., rot:].cpu(), x[..., rot:])
    assert wb.last_launch_count() == 1


@pytest.mark.gpu
@pytest.mark.parametrize("rot", [128, 48])
def test_rope_in_place_and_strided(rot):
    x = torch.randn((4, 50, 3, 136), dtype=torch.bfloat16, device="cuda")
    freqs, _ = wb.rope_freqs(rot)
    positions = torch.arange(50, dtype=torch.int32, device="cuda") * 3
    q, k = x[:, :, 0, :128], x[:, :, 1, 8:]
    want, want_k = wb.rope(q, positions, freqs, k=k)
    before = x.clone()
    got, got_k = wb.rope(q, positions, freqs, k=k, q_out=q, k_out=k)
    assert got.data_ptr() == q.data_ptr() and torch.equal(got, want) and torch.equal(got_k, want_k)
    assert torch.equal(x[:, :, 2], before[:, :, 2]) and torch.equal(x[:, :, 0, 128:], before[:, :, 0, 128:])
    # an odd offset: no wide vectors, the same numbers
    y = torch.zeros((4, 50, 131), dtype=torch.bfloat16, device="cuda")
    odd, _ = wb.rope(before[:, :, 0, :128], positions, freqs, q_out=y[..., 3:])
    assert torch.equal(odd, want)


@pytest.mark.gpu
def test_rope_gradient_is_the_inverse():
    # <g, R x> = <R' g, x> for the formula's own R, and against differences: R is linear, so a difference quotient has no
    # error but rounding
    freqs, amplitude = wb.rope_freqs(32, scaling="parts", factor=4.0, trained_len=512)
    positions = torch.arange(900, 911, dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    x, dy = (torch.randn((2, 11, 40), device="cuda", generator=g) for _ in range(2))
    for inter in (False, True):
        kw = dict(interleaved=inter, amplitude=amplitude)
        y, _ = wb.rope(x, positions, freqs, **kw)
        dx, _ = wb.rope(dy, positions, freqs, inverse=True, **kw)
        size = float((dy.abs().double().sum()) * x.abs().max())
        assert abs(float((dy.double() * y.double()).sum() - (dx.double() * x.double()).sum())) <= 16 * 2.0 ** -24 * size
        for at in ((0, 3, 5), (1, 10, 31), (1, 0, 39)):
            step = torch.zeros_like(x)
            step[at] = 1.0
            up, _ = wb.rope(x + step, positions, freqs, **kw)
            slope = float((dy.double() * (up.double() - y.double())).sum())
            # x + 1 is rounded, and y and up to 8 units of the two channels that change
            assert abs(slope - float(dx[at])) <= 64 * 2.0 ** -24 * float(dy[at[0], at[1]].abs().max()) * 6


@pytest.mark.gpu
def test_rope_no_tokens():
    freqs, _ = wb.rope_freqs(8)
    q, _ = wb.rope(torch.empty((3, 0, 8), device="cuda"), torch.empty((1, 0), dtype=torch.int32, device="cuda"), freqs)
    assert q.shape == (3, 0, 8) and wb.last_launch_count() == 0


APPENDS = [
    # new, own, prefix, q heads, kv heads, dim, rot, page, type, interleaved, axes (0: positions left out), token-major cache
    ([1], [1], 0, 1, 1, 64, 64, 16, "bf16", False, 0, False),
    ([1] * 40, [1 + 7 * i for i in range(40)], 1000, 8, 2, 128, 128, 16, "bf16", False, 0, False),
    ([3, 0, 50, 17], [3, 5, 90, 100], 77, 6, 3, 64, 32, 32, "fp16", True, 3, True),
    ([200, 1], [333, 16], 12345, 2, 2, 128, 128, 128, "bf16", True, 0, True),
    ([9], [20], 3, 0, 2, 96, 40, 16, "fp16", False, 1, False),
    ([5, 6], [6, 7], 0, 0, 2, 20, 0, 64, "bf16", False, 0, False),     # no rotation
    ([4, 3], [40, 30], 9, 3, 1, 33, 6, 16, "bf16", True, 0, True),     # odd head_dim
]


@pytest.mark.gpu
@pytest.mark.parametrize("case", APPENDS, ids=range(len(APPENDS)))
def test_append_matches_definition(case):
    new, own, prefix, qh, kh, dim, rot, page, kind, inter, axes, token_major = case
    dtype = TYPES[kind]
    g = torch.Generator().manual_seed(dim + len(new))
    tokens = sum(new) + 2                                        # two tokens of no sequence at the end
    need = [-(-n // page) for n in own]
    pages = sum(need) + 2
    order = torch.randperm(pages, generator=g)
    table = torch.full((len(new), max(need) + 1), -5, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    q = torch.randn((tokens, max(qh, 1), dim), generator=g).to(dtype).transpose(0, 1)
    k, v = (torch.randn((tokens, kh, dim), generator=g).to(dtype).transpose(0, 1) for _ in range(2))
    shape = (pages, page, kh, dim) if token_major else (pages, kh, page, dim)
    view = (lambda t: t.transpose(1, 2)) if token_major else (lambda t: t)
    kc, vc = (view(torch.randn(shape, generator=g).to(dtype)) for _ in range(2))
    places = [have - n + i for n, have in zip(new, own) for i in range(n)] + [0, 0]
    whose = [b for b, n in enumerate(new) for _ in range(n)]
    positions = torch.tensor(places)[None] + prefix
    split = [rot // 2] if axes < 2 else axes_of(rot // 2, axes)
    if axes:
        positions = torch.stack([torch.tensor(places) * (a + 2) + a for a in range(axes)])
    freqs = wb.rope_freqs(rot, device="cpu")[0] if rot else None
    cache = wb.PagedCache(view(view(kc).contiguous().cuda()), view(view(vc).contiguous().cuda()))
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    q_out = torch.full_like(q, 9.0).cuda() if qh else None
    wb.cache_append(cache, k.cuda(), v.cuda(), torch.tensor([0] + new).cumsum(0).to(torch.int32).cuda(),
                    torch.tensor(own, dtype=torch.int32).cuda(), table.cuda(), positions=positions.to(torch.int32).cuda() if axes else None,
                    freqs=None if freqs is None else freqs.cuda(), q=q.cuda() if qh else None, q_out=q_out, prefix_len=prefix,
                    interleaved=inter, axis_pairs=split if rot else None, amplitude=0.75, dev_status=status)
    assert status.tolist() == [0] * 4 and wb.last_launch_count() == 1
    turn = (lambda x: rotated(x.double(), positions, radians(freqs), split, inter, 0.75)) if rot else (lambda x: x.double())
    kr = turn(k)
    want_k, want_v = kc.double().clone(), vc.double().clone()
    size = torch.zeros_like(want_k)
    tol, unit = rotation_tolerance(k.double(), rot, inter, 0.75, dtype)
    for t, b in enumerate(whose):
        to = int(table[b, places[t] // page])
        want_k[to, :, places[t] % page], want_v[to, :, places[t] % page] = kr[:, t], v[:, t].double()
        size[to, :, places[t] % page] = tol[:, t] + unit * kr[:, t].abs() + 2.0 ** -25
    assert bool(((cache.k.double().cpu() - want_k).abs() <= size).all())
    assert torch.equal(cache.v.double().cpu(), want_v)
    if qh:
        live = len(whose)
        close(q_out[:, :live], turn(q)[:, :live], q.double()[:, :live], rot, inter, 0.75, dtype)
        assert bool((q_out[:, live:] == 9).all())


@pytest.mark.gpu
def test_append_reports_what_is_malformed_and_writes_the_rest():
    freqs, _ = wb.rope_freqs(64)
    for what, site in (("page", 42), ("short", 41), ("long", 41), ("start", 40)):
        kc = torch.zeros((8, 1, 16, 64), dtype=torch.bfloat16, device="cuda")
        cache = wb.PagedCache(kc, torch.zeros_like(kc))
        k = torch.ones((1, 6, 64), dtype=torch.bfloat16, device="cuda")
        start = torch.tensor([0, 2, 4, 6], dtype=torch.int32, device="cuda")
        lens = torch.tensor([2, 4, 10], dtype=torch.int32, device="cuda")
        table = torch.tensor([[0], [1], [2]], dtype=torch.int32, device="cuda")
        if what == "page":
            table[1, 0] = 8
        elif what == "short":
            lens[1] = 1
        elif what == "long":
            lens[1] = 17
        else:
            start[1] = -1
        status = torch.zeros(4, dtype=torch.int32, device="cuda")
        wb.cache_append(cache, k, k, start, lens, table, freqs=freqs, dev_status=status)
        status = status.tolist()
        assert status[0] == wb.ERR_BAD_MASK and status[1] == site, (what, status)
        slots = cache.v[:, 0, :, 0].cpu() != 0
        want = torch.zeros((8, 16), dtype=torch.bool)
        want[2, 8:10] = True
        if what != "start":
            want[0, 0:2] = True
        assert torch.equal(slots, want), what


@pytest.mark.gpu
def test_append_beyond_32_bits():
    # 2^25 elements a page, 72 pages: the last one begins at 2.4e9 elements
    k = torch.zeros((72, 8, 65536, 64), dtype=torch.bfloat16, device="cuda")
    cache = wb.PagedCache(k, torch.zeros_like(k))
    x = torch.randn((8, 3, 64), dtype=torch.bfloat16, device="cuda")
    start, lens = torch.tensor([0, 3], dtype=torch.int32, device="cuda"), torch.tensor([65536], dtype=torch.int32, device="cuda")
    wb.cache_append(cache, x, x, start, lens, torch.tensor([[71]], dtype=torch.int32, device="cuda"))
    assert torch.equal(cache.k[71, :, 65533:], x) and torch.equal(cache.v[71, :, 65533:], x)
    assert int(torch.count_nonzero(cache.k)) == int(torch.count_nonzero(x))


def append_ones(starts, tokens, lens, prefix=0, k=None, page=16):
    """keys and values of ones (or k) into pages b of sequence b; returns (status, slots that were written, cache)"""
    batch = len(lens)
    kc = torch.zeros((batch, 1, page, 64), dtype=torch.bfloat16, device="cuda")
    cache = wb.PagedCache(kc, torch.zeros_like(kc))
    x = torch.ones((1, tokens, 64), dtype=torch.bfloat16, device="cuda") if k is None else k
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    wb.cache_append(cache, x, x, torch.tensor(starts, dtype=torch.int32, device="cuda"), torch.tensor(lens, dtype=torch.int32, device="cuda"),
                    torch.arange(batch, dtype=torch.int32, device="cuda")[:, None], freqs=wb.rope_freqs(64)[0], prefix_len=prefix, dev_status=status)
    return status.tolist(), cache.v[:, 0, :, 0].cpu() != 0, cache


@pytest.mark.gpu
@pytest.mark.parametrize("starts, tokens, lens", [([5, 8, 10], 10, [4, 2]), ([3, 3], 3, [2]), ([4, 4, 4], 9, [1, 2]), ([1000, 1001], 1001, [7])])
def test_append_leaves_tokens_in_front_of_the_first_sequence_alone(starts, tokens, lens):
    status, slots, _ = append_ones(starts, tokens, lens)
    assert status == [0] * 4
    want = torch.zeros_like(slots)
    for b, n in enumerate(lens):
        want[b, n - (starts[b + 1] - starts[b]):n] = True
    assert torch.equal(slots, want)


@pytest.mark.gpu
@pytest.mark.parametrize("starts, tokens, bad", [
    ([0, 6, 4, 6], 6, [(1, 4)]), ([0, 3, 9], 6, [(1, 9)]), ([0, 2, -3, 4, 6], 6, [(1, -3), (2, -3)]), ([6, 0, 6], 6, [(0, 0)]),
    ([0] * 700 + [1, 0, 2], 2, [(700, 0)]),                       # more sequences than threads of a block, in one block
    (list(range(4000)) + [0], 3999, [(3999, 0)]),                 # several blocks
])
def test_append_reports_starts_that_decrease_or_leave_the_tensors(starts, tokens, bad):
    status, slots, _ = append_ones(starts, tokens, [16] * (len(starts) - 1))
    assert status in [[wb.ERR_BAD_MASK, 40, b, value] for b, value in bad]
    for b, (lo, hi) in enumerate(zip(starts, starts[1:])):
        if lo < 0 or hi < lo or hi > tokens:
            assert not bool(slots[b].any()), b                    # counts as having no new tokens


@pytest.mark.gpu
def test_append_positions_beyond_31_bits():
    # prefix_len + place passes 2^31 - 1: the positions go on, they do not turn negative
    prefix, n = 2 ** 31 - 5, 12
    k = torch.randn((1, n, 64), generator=torch.Generator().manual_seed(1)).bfloat16()
    status, _, cache = append_ones([0, n], n, [n], prefix, k.cuda())
    assert status == [0] * 4
    positions = prefix + torch.arange(n)[None]
    want = rotated(k.double(), positions, radians(wb.rope_freqs(64)[0]), [32], False)
    # (the definition's angle is a product of 2^31 and a table entry in 64 bits: off by 2^-53 of 2^31 radians, 2^-22)
    tol, unit = rotation_tolerance(k.double(), 64, False, 1.0, torch.bfloat16)
    size = (k.double().abs() + k.double().abs().roll(32, -1)) * 2.0 ** -21
    got = cache.k[0, :, :n].double().cpu()
    assert bool(((got - want).abs() <= tol + size + unit * want.abs()).all())
