"""Host-only checks of prompt attention and of the page calls: outputs over inputs, sizes whose loops would not end.  A call that is not refused
ends where it asks for the device (ERR_CUDA), so these tests run on machines without one alone: the addresses are made up."""
import ctypes
import itertools
import random

import pytest
import torch

from paper_2609_34814_b200 import binding as wb
from paper_2609_34814_b200 import build as wbuild


pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses must not reach a device")


@pytest.fixture(scope="module")
def lib():
    wbuild.build()
    return wb.load()


BASE = 1 << 32
TAKEN = wb.ERR_CUDA


def prompt(lib, heads, kv_heads, tokens, dim, at, strides):
    """The status of a call whose q, k, v and o lie `at` elements behind BASE."""
    d = wb.PromptDesc(1, tokens, heads, kv_heads, dim, wb.BF16, 0, *strides)
    q, k, v, o = (BASE + 2 * a for a in at)
    return lib.waveal_prompt_attn(ctypes.byref(d), q, k, v, o, None, BASE - 4096, None, 0.0, BASE - (1 << 30), 1 << 29, None, None)


@pytest.mark.parametrize("heads, kv_heads, tokens, dim", [(8, 2, 100, 128), (1, 1, 1, 64), (4, 4, 1, 64), (1, 1, 300, 64), (128, 1, 77, 64), (2, 2, 3000, 128)])
@pytest.mark.parametrize("order", ["nhd", "hnd"])
def test_prompt_results_beside_their_inputs(lib, heads, kv_heads, tokens, dim, order):
    """One buffer for all four tensors, each row of a token (or head) holding q, k, v and o in turn: none of them meets another.  o moved by 8 elements
    either way meets its neighbour, unless there is none."""
    parts = [heads, kv_heads, kv_heads, heads]
    if order == "nhd":
        begin = [0] + list(itertools.accumulate(p * dim for p in parts))
        at, strides = begin[:4], [(dim, begin[4])] * 4
        end = begin[4]
    else:
        begin = [0] + list(itertools.accumulate(p * dim * tokens for p in parts))
        at, strides = begin[:4], [(dim * tokens, dim)] * 4
        end = begin[4]
    assert prompt(lib, heads, kv_heads, tokens, dim, at, strides) == TAKEN
    # into v's last head; far behind; into the next token's q (where there is one)
    assert prompt(lib, heads, kv_heads, tokens, dim, at[:3] + [at[3] - 8], strides) == wb.ERR_INVALID_ARG
    assert prompt(lib, heads, kv_heads, tokens, dim, at[:3] + [end * tokens], strides) == TAKEN
    into_q = wb.ERR_INVALID_ARG if order == "nhd" and tokens > 1 else TAKEN
    assert prompt(lib, heads, kv_heads, tokens, dim, at[:3] + [at[3] + 8], strides) == into_q
    # o over the last row alone of each input, and just behind it
    for i, h in enumerate((heads, kv_heads, kv_heads)):
        last = at[i] + (h - 1) * strides[i][0] + (tokens - 1) * strides[i][1]
        assert prompt(lib, heads, kv_heads, tokens, dim, at[:3] + [last], strides) == wb.ERR_INVALID_ARG


def test_prompt_results_over_an_input_in_part(lib):
    """Tensors by themselves, o beginning inside one of them."""
    heads, kv_heads, tokens, dim = 8, 2, 100, 128
    strides = [(dim, heads * dim), (dim, kv_heads * dim), (dim, kv_heads * dim), (dim, heads * dim)]
    size = [heads * tokens * dim, kv_heads * tokens * dim, kv_heads * tokens * dim]
    at = [10_000_000, 20_000_000, 30_000_000, 40_000_000]
    assert prompt(lib, heads, kv_heads, tokens, dim, at, strides) == TAKEN
    for i in range(3):
        for o, status in ((at[i] + size[i] - 8, wb.ERR_INVALID_ARG), (at[i] + size[i], TAKEN), (at[i] - heads * tokens * dim + 8, wb.ERR_INVALID_ARG), (at[i] - heads * tokens * dim, TAKEN), (at[i] + 8, wb.ERR_INVALID_ARG)):
            assert prompt(lib, heads, kv_heads, tokens, dim, at[:3] + [o], strides) == status, (i, o)


def test_prompt_overlap_against_sets(lib):
    """Random views of a small buffer: what is let through has no element in common, and with equal strides what is refused has one."""
    r = random.Random(5)
    dim, met, let = 64, 0, 0
    for _ in range(3000):
        heads, tokens = r.choice([(1, 1), (2, 1), (1, 5), (2, 3), (4, 3), (3, 2)])
        kv_heads = r.choice([h for h in (1, 2, 3, 4) if heads % h == 0])
        a, b = r.randint(8, 40) * 8, r.randint(8, 40) * 8
        same = (a, a * heads + 8 * r.randint(0, 30)) if r.random() < 0.5 else (b * tokens + 8 * r.randint(0, 30), b)
        strides = [same, (a, 2048), (a, 2048), same]
        at = [r.randint(0, 100) * 8, 1_000_000, 2_000_000, r.randint(0, 300) * 8]

        def elements(at, heads, stride):
            return {at + h * stride[0] + t * stride[1] + c for h in range(heads) for t in range(tokens) for c in range(0, dim, 8)}
        common = bool(elements(at[0], heads, same) & elements(at[3], heads, same))
        assert prompt(lib, heads, kv_heads, tokens, dim, at, strides) == (wb.ERR_INVALID_ARG if common else TAKEN), (heads, tokens, same, at)
        met, let = met + common, let + (not common)
    assert met > 300 and let > 300


def test_prompt_overlap_with_one_stride_in_common(lib):
    """The same where head strides differ (repeated heads with a stride of 0 among them), or token strides: still exact."""
    r = random.Random(7)
    dim, met, let = 64, 0, 0
    for _ in range(6000):
        heads, tokens = r.choice([(2, 1), (2, 3), (4, 3), (3, 2), (6, 5), (4, 9)])
        kv_heads = r.choice([h for h in (1, 2, 3, 4, 6) if heads % h == 0])
        if r.random() < 0.6:
            common = 8 * r.randint(0, 300)
            k = (r.choice([0, 64, 128, 8 * r.randint(0, 60)]), common)
            o = (64 + 8 * r.randint(0, 30), max(common, 8))
            common = o[1]
            k = (k[0], common)
        else:
            common = 64 + 8 * r.randint(0, 300)
            k = (common, r.choice([0, 64, 8 * r.randint(0, 60)]))
            o = (common, 64 + 8 * r.randint(0, 30))
        rows = sorted(h * o[0] + t * o[1] for h in range(heads) for t in range(tokens))
        if any(b - a < dim for a, b in zip(rows, rows[1:])):
            continue                                                      # o over itself is refused before

        def elements(at, heads, stride):
            return {at + h * stride[0] + t * stride[1] + c for h in range(heads) for t in range(tokens) for c in range(0, dim, 8)}
        at = [5_000_000, 8 * r.randint(0, 200), 2_000_000, 8 * r.randint(0, 400)]
        meets = bool(elements(at[1], kv_heads, k) & elements(at[3], heads, o))
        got = prompt(lib, heads, kv_heads, tokens, dim, at, [(64, 64 * heads), k, (64, 64 * kv_heads), o])
        assert got == (wb.ERR_INVALID_ARG if meets else TAKEN), (heads, kv_heads, tokens, at, k, o)
        met, let = met + meets, let + (not meets)
    assert met > 500 and let > 500


def test_prompt_overlap_of_the_largest(lib):
    """Two strides in common, one, none: 10^9 rows are decided about without a walk through all of them."""
    heads = tokens = 31000
    row = 128 * heads
    strides = lambda k, o: [(128, row), k, (128, row), o]  # noqa: E731
    far = 1 << 45
    for k, o, at, status in (((128, 2 * row), (128, 2 * row), row, TAKEN), ((128, 2 * row), (128, 2 * row), row - 8, wb.ERR_INVALID_ARG),
                             # (o's heads fill the second half of every 2 * row elements, the repeated key head is at the front of the first)
                             ((0, 2 * row), (128, 2 * row), row, TAKEN), ((0, 2 * row), (128, 2 * row), 0, wb.ERR_INVALID_ARG),
                             ((136, 4 * row), (128, 2 * row), 0, wb.ERR_INVALID_ARG), ((136, 4 * row), (128, 2 * row), 1 << 44, TAKEN)):
        assert prompt(lib, heads, heads, tokens, 128, [far, 0, 2 * far, at], strides(k, o)) == status, (k, o, at)
    # three heads a token that read one repeated key head
    assert prompt(lib, 3, 3, 1 << 24, 64, [far, 0, 2 * far, 64], [(64, 192), (0, 256), (64, 192), (64, 256)]) == TAKEN


def pool(n_pages=10, head_dim=128):
    return wb.CacheDesc(n_pages, 16, 2, head_dim, wb.BF16, (32 * head_dim, 16 * head_dim, head_dim), (32 * head_dim, 16 * head_dim, head_dim))


MOST = 1 << 30
LAST = (1 << 31) - 1


@pytest.mark.parametrize("over", [MOST + 1, LAST - 16384, LAST])
def test_sizes_whose_loops_would_run_over(lib, over):
    """Loops over rows, a row's entries and the pool's pages go on in steps of up to 2^14 with 32-bit counters: from 2^31 - 2^14 on they would come back
    negative.  Sizes up to 2^30 are taken."""
    n = ctypes.c_size_t(0)
    at = [BASE + (i << 34) for i in range(10)]
    ws, room = BASE + (20 << 34), 1 << 40

    def fork(cache, *sizes):
        d = wb.ForkDesc(*sizes)
        status = lib.waveal_cache_fork(ctypes.byref(cache), ctypes.byref(d), *at, ws, room, None, None)
        query = lib.waveal_cache_fork_workspace_bytes(ctypes.byref(cache), ctypes.byref(d), ctypes.byref(n))
        assert query == (wb.OK if status == TAKEN else status)
        return status

    def compact(cache, *sizes):
        return lib.waveal_cache_compact(ctypes.byref(cache), ctypes.byref(wb.CompactDesc(*sizes)), *at, ws, room, None)
    for n_pages, sizes in ((over, (1, 1, 1, 1, 1, 1)), (10, (over, 1, 0, 1, 0, 1)), (10, (1, over, 1, 0, 1, 0)), (10, (1, 1, over, 1, over, 1)),
                           (10, (1, 1, 1, over, 1, over))):
        assert fork(pool(n_pages), *sizes) == wb.ERR_UNSUPPORTED, sizes
        assert fork(pool(min(n_pages, MOST)), *(min(x, MOST) for x in sizes)) == TAKEN, sizes
    for n_pages, sizes in ((over, (1, 1, 1, 1, 1)), (10, (over, 0, 0, 0, 0)), (10, (1, over, 0, over, over))):
        assert compact(pool(n_pages), *sizes) == wb.ERR_UNSUPPORTED, sizes
        assert compact(pool(min(n_pages, MOST)), *(min(x, MOST) for x in sizes)) == TAKEN, sizes
    assert lib.waveal_cache_compact_workspace_bytes(ctypes.byref(pool(over)), ctypes.byref(n)) == wb.ERR_UNSUPPORTED
    assert lib.waveal_cache_compact_workspace_bytes(ctypes.byref(pool(MOST)), ctypes.byref(n)) == wb.OK


def test_prompt_results_over_each_other(lib):
    """Strides of o by which two of its rows have an element in common are refused, all others taken."""
    r, met, let = random.Random(6), 0, 0
    for _ in range(4000):
        heads, tokens, dim = r.randint(1, 6), r.randint(1, 6), r.choice([64, 128])
        stride = [r.choice([0, 8, dim - 8, dim, dim + 8, r.randint(0, 100) * 8, dim * r.randint(1, 6)]) for _ in range(2)]
        rows = sorted(h * stride[0] + t * stride[1] for h in range(heads) for t in range(tokens))
        common = any(b - a < dim for a, b in zip(rows, rows[1:]))
        strides = [(dim, heads * dim), (dim, dim), (dim, dim), stride]
        d = wb.PromptDesc(1, tokens, heads, 1, dim, wb.BF16, 0, *map(tuple, strides))
        n = ctypes.c_size_t(0)
        assert lib.waveal_prompt_attn_workspace_bytes(ctypes.byref(d), ctypes.byref(n)) == (wb.ERR_INVALID_ARG if common else wb.OK), (heads, tokens, dim, stride)
        met, let = met + common, let + (not common)
    assert met > 500 and let > 500
    # the largest: 10^9 rows, heads and tokens as many (a token's heads reach 30,999 * 128 + 128 = 31,000 * 128 elements far)
    for stride, status in (((128, 128 * 31000 + 8), wb.OK), ((128, 128 * 31000 - 8), wb.ERR_INVALID_ARG), ((136, 128 * 31000 + 8), wb.ERR_INVALID_ARG), ((1 << 40, 128), wb.OK), ((128, 1 << 40), wb.OK), ((0, 1 << 62), wb.ERR_INVALID_ARG)):
        d = wb.PromptDesc(1, 31000, 31000, 31000, 128, wb.BF16, 0, (128, 128), (128, 128), (128, 128), stride)
        assert lib.waveal_prompt_attn_workspace_bytes(ctypes.byref(d), ctypes.byref(ctypes.c_size_t(0))) == status, stride
