"""Copying, forking and compacting pages against their definitions on lists: whole numbers and moved bits are equal, not near."""
import random

import pytest
import torch

from paper_2609_34814_b200 import binding as wb
from pages_util import Pool, compacted, forked, ints, on_gpu, up

pytestmark = pytest.mark.gpu

NO_ERROR = [0, 0, 0, 0]


def fork(pool, parents, keep, room, max_pages=None, offset=0):
    k, v = on_gpu(pool.k, offset), on_gpu(pool.v, offset)
    status = ints(NO_ERROR)
    wide = max([up(max(n, m), pool.page) for n, m in zip(keep, room)] + [1]) if max_pages is None else max_pages
    table, refs = wb.cache_fork(wb.PagedCache(k, v), ints(pool.padded(), (pool.rows, pool.wide)), ints(pool.held), ints(pool.refs), ints(keep), ints(room),
                                parents=None if parents is None else ints(parents), max_pages=wide, dev_status=status)
    return table, refs, k, v, status


def check(pool, parents, keep, room, offset=0):
    table, refs, k, v, status = fork(pool, parents, keep, room, offset=offset)
    rows, counts, copies = forked(pool.table, pool.held, pool.refs, keep, room, list(range(pool.rows)) if parents is None else parents, pool.page)
    want_k, want_v = pool.k.clone(), pool.v.clone()
    for a, b, n in copies:
        want_k[b, :, :n], want_v[b, :, :n] = pool.k[a, :, :n], pool.v[a, :, :n]
    want = [r + [-1] * (table.shape[1] - len(r)) for r in rows]
    assert status.tolist() == NO_ERROR
    assert table.tolist() == want
    assert refs.tolist() == counts
    assert torch.equal(k.cpu(), want_k) and torch.equal(v.cpu(), want_v)
    return copies


def wishes(pool, rows, seed, grow=50):
    r = random.Random(seed)
    parents = [r.choice([-1] + list(range(pool.rows)) * 3) for _ in range(rows)]
    keep = [0 if p < 0 else r.choice([pool.held[p], r.randint(0, pool.held[p])]) for p in parents]
    return parents, keep, [n + r.choice([0, 1, r.randint(0, grow)]) for n in keep]


@pytest.mark.parametrize("rows, most, page, new_rows, kw", [
    (1, 0, 16, 1, {}), (1, 1, 16, 1, {}), (1, 16, 16, 3, {}), (1, 17, 16, 2, {}), (5, 100, 16, 5, {}), (5, 100, 32, 40, {}), (40, 300, 16, 3, {}),
    (7, 500, 64, 9, dict(token_major=True)), (6, 1000, 256, 30, dict(heads=5, dim=128)), (9, 300, 16, 12, dict(heads=1, dim=96, dtype=torch.float16)),
    (9, 300, 32, 12, dict(heads=3, dim=20)), (4, 200, 16, 12, dict(dim=2, heads=1)), (300, 900, 16, 350, dict(heads=1)), (1500, 60, 16, 1400, dict(heads=1, dim=8)),
    (3, 30000, 16, 6, dict(heads=1, dim=8)), (64, 9000, 16, 64, dict(heads=1, dim=8)), (200, 9000, 16, 210, dict(heads=1, dim=8)),
    (600, 9000, 16, 500, dict(heads=1, dim=8)), (4, 200, 16, 12, dict(heads=1, dim=8, spare=800.0)), (4, 200, 16, 12, dict(heads=1, dim=8, spare=4000.0)),
    (4, 200, 16, 12, dict(heads=1, dim=8, spare=15000.0)), (30, 2000, 16, 33, dict(heads=1, dim=8, spare=2.0))])
def test_fork(rows, most, page, new_rows, kw):
    pool = Pool(rows, most, page=page, seed=rows + most, **{"spare": 3.0 if new_rows > rows else 1.5, **kw})
    free = sum(n == 0 for n in pool.refs)
    for seed in range(3):
        parents, keep, room = wishes(pool, new_rows, seed)
        while sum(up(m, page) for m in room) > free:               # fits whatever is shared
            parents = parents[:-1] if len(parents) > 1 else [-1]
            keep, room = keep[:len(parents)], room[:len(parents)]
            if parents == [-1]:
                keep, room = [0], [0]
        check(pool, parents, keep, room)


def test_fork_without_parents_goes_on():
    pool = Pool(16, 1000, seed=3, shared=0.0)
    assert check(pool, None, pool.held, [n + 1 for n in pool.held]) == []      # every row keeps its last page


def test_every_row_from_one():
    pool = Pool(1, 23, page=16, spare=30.0, seed=4, outside=0.0)
    copies = check(pool, [0] * 20, [23] * 20, [40] * 20)
    assert len(copies) == 19 and {a for a, _, _ in copies} == {pool.table[0][1]}


def test_a_page_held_from_outside_is_copied():
    pool = Pool(2, 40, page=16, spare=4.0, seed=5, shared=0.0, outside=0.0)
    last = pool.table[0][pool.held[0] // 16]
    pool.refs[last] += 1
    copies = check(pool, [0, 1], pool.held, [n + 3 for n in pool.held])
    assert (last, pool.held[0] % 16) in [(a, n) for a, _, n in copies]


def test_cut_back_into_a_page_that_another_row_fills():
    pool = Pool(1, 64, page=16, spare=8.0, seed=6, outside=0.0)
    # row 0 goes on whole, row 1 keeps 20 tokens: its second page is full in row 0
    copies = check(pool, [0, 0, 0], [64, 20, 25], [64, 40, 25])
    assert sorted(n for _, _, n in copies) == [4, 9]
    # nobody fills it: the first of those that end in it keeps it
    copies = check(pool, [0, 0], [25, 20], [25, 20])
    assert [n for _, _, n in copies] == [4]


@pytest.mark.parametrize("offset", [1, 4])
def test_fork_unaligned(offset):
    pool = Pool(5, 100, seed=7, spare=4.0)
    check(pool, [0, 0, 1, 2, 4], [pool.held[p] for p in (0, 0, 1, 2, 4)], [pool.held[p] + 20 for p in (0, 0, 1, 2, 4)], offset=offset)


def test_all_rows_end_and_no_rows():
    pool = Pool(12, 300, seed=8)
    check(pool, [-1] * 4, [0] * 4, [9] * 4)
    cache = wb.PagedCache(on_gpu(pool.k), on_gpu(pool.v))
    none = ints([])
    table, refs = wb.cache_fork(cache, ints(pool.padded()), ints(pool.held), ints(pool.refs), none, none, parents=none)
    assert table.shape == (0, pool.wide)
    assert refs.tolist() == forked(pool.table, pool.held, pool.refs, [], [], [], 16)[1]
    # the first rows of all
    table, refs = wb.cache_fork(cache, ints([]).view(0, 0), none, refs, ints([0, 0]), ints([20, 1]), parents=ints([-1, -1]), max_pages=2)
    assert table.tolist() == [[-1, -1], [-1, -1]]


def test_strided_tables_and_given_outputs():
    pool = Pool(6, 200, seed=9, spare=4.0)
    old = torch.full((6, pool.wide + 5), 99, dtype=torch.int32, device="cuda")
    old[:, :pool.wide] = ints(pool.padded())
    out = torch.full((6, 40), 77, dtype=torch.int32, device="cuda")
    refs_out = torch.empty_like(ints(pool.refs))
    cache = wb.PagedCache(on_gpu(pool.k), on_gpu(pool.v))
    room = [n + 30 for n in pool.held]
    table, refs = wb.cache_fork(cache, old[:, :pool.wide], ints(pool.held), ints(pool.refs), ints(pool.held), ints(room), table_out=out[:, 3:30], refs_out=refs_out)
    rows, counts, _ = forked(pool.table, pool.held, pool.refs, pool.held, room, range(6), 16)
    assert table.tolist() == [r + [-1] * (27 - len(r)) for r in rows] and refs_out.tolist() == counts and refs is refs_out
    assert (out[:, :3] == 77).all() and (out[:, 30:] == 77).all()


def test_out_of_pages():
    pool = Pool(4, 100, seed=10, spare=0.0, outside=0.0)
    free = sum(n == 0 for n in pool.refs)
    room = [n + 16 * free for n in pool.held]
    table, refs, k, v, status = fork(pool, None, pool.held, room)
    rows, counts, _ = forked(pool.table, pool.held, pool.refs, pool.held, room, range(4), 16)
    assert table.tolist() == [r + [-1] * (table.shape[1] - len(r)) for r in rows] and refs.tolist() == counts
    short = next(b for b, r in enumerate(rows) if -1 in r)
    assert status.tolist() == [wb.ERR_NO_PAGES, 85, short, sum(r.count(-1) for r in rows)]
    assert min(counts) == 1


def test_a_copy_that_finds_no_page():
    pool = Pool(1, 20, page=16, spare=0.0, seed=11, outside=0.0)
    free = sum(n == 0 for n in pool.refs)
    table, refs, k, v, status = fork(pool, [0] * (free + 2), [20] * (free + 2), [20] * (free + 2))
    assert table[:free + 1].min() >= 0 and table[free + 1].tolist() == [pool.table[0][0], -1]
    assert status.tolist() == [wb.ERR_NO_PAGES, 85, free + 1, 1]


@pytest.mark.parametrize("what, site, row, value", [("parent", 80, 2, 5), ("held", 81, 1, -3), ("held far", 81, 1, 1000), ("keep", 82, 3, 51), ("keep below", 82, 3, -1),
                                                    ("room", 83, 0, 161), ("entry", 84, 1, -2), ("entry far", 84, 1, 10 ** 9), ("last entry", 84, 1, -2)])
def test_malformed(what, site, row, value):
    pool = Pool(5, 50, seed=12, shared=0.0, outside=0.0, spare=6.0, wide=10)
    pool.held = [50] * 5
    pool.table = [list(range(4 * b, 4 * b + 4)) for b in range(5)]
    pool.refs = [1] * 20 + [0] * (pool.n_pages - 20)
    parents, keep, room, held, table = list(range(5)), [50] * 5, [60] * 5, list(pool.held), [list(r) for r in pool.padded()]
    empty, lost = row, None
    if what == "parent":
        parents[2] = 5
    elif what.startswith("held"):
        held[1] = value
        keep[1] = 0                                                   # of nothing
        empty = None
    elif what.startswith("keep"):
        keep[3] = value
    elif what == "room":
        room[0] = 161
    else:
        lost = 3 if what == "last entry" else 1
        table[1][lost] = value
        empty = None
    k, v = on_gpu(pool.k), on_gpu(pool.v)
    status = ints(NO_ERROR)
    out, refs = wb.cache_fork(wb.PagedCache(k, v), ints(table), ints(held), ints(pool.refs), ints(keep), ints(room), parents=ints(parents), dev_status=status)
    assert status.tolist() == [wb.ERR_BAD_MASK, site, row, value]
    out = out.tolist()
    for b in range(5):
        if b == empty:
            assert out[b] == [-1] * 10
        elif what.startswith("held") and b == 1:
            assert sorted(out[1][:4]) == out[1][:4] and out[1][4:] == [-1] * 6      # room alone; its old pages are not given back
        elif lost is not None and b == 1:
            assert out[1][:4] == [-1 if j == lost else 4 + j for j in range(4)]
        else:
            assert out[b][:4] == pool.table[b] and out[b][4:] == [-1] * 6
    assert torch.equal(k.cpu(), pool.k)
    counted = [0] * pool.n_pages
    for r in out:
        for p in r:
            if p >= 0:
                counted[p] += 1
    if what.startswith("held"):
        counted = [n + (4 <= p < 8) for p, n in enumerate(counted)]                 # nobody let go of these
    if lost is not None:
        counted[4 + lost] += 1
    assert refs.tolist() == counted


@pytest.mark.parametrize("rows, most, page, spare, kw", [
    (1, 1, 16, 0.0, {}), (3, 100, 16, 0.5, {}), (3, 100, 16, 20.0, {}), (40, 400, 32, 1.0, dict(token_major=True)), (9, 3000, 256, 0.7, dict(heads=3, dim=128)),
    (20, 300, 16, 1.0, dict(heads=3, dim=20)), (500, 900, 16, 0.3, dict(heads=1, dim=8)), (300, 9000, 16, 2.0, dict(heads=1, dim=8)), (5, 100, 16, 1.0, dict(offset=1)),
    (60, 900, 16, 1.5, dict(heads=1, dim=8)), (60, 900, 16, 3.0, dict(heads=1, dim=8, offset=1)), (150, 900, 16, 5.0, dict(heads=1, dim=8, offset=1))])
def test_compact(rows, most, page, spare, kw):
    offset = kw.get("offset", 0)
    pool = Pool(rows, most, page=page, spare=spare, seed=rows + page, **kw)
    place, after, n = compacted(pool.refs)
    k, v = on_gpu(pool.k, offset), on_gpu(pool.v, offset)
    r = wb.cache_compact(wb.PagedCache(k, v), ints(pool.refs), page_table=ints(pool.padded()), prefix_pages=ints(pool.prefix + [-1, pool.n_pages]))
    assert r.used.tolist() == [n] and r.place.tolist() == place and r.page_refs.tolist() == after
    assert r.page_table.tolist() == [[place[p] for p in row] + [-1] * (pool.wide - len(row)) for row in pool.table]
    assert r.prefix_pages.tolist() == [place[p] for p in pool.prefix] + [-1, -1]
    want_k, want_v = pool.k.clone(), pool.v.clone()
    for a, b in enumerate(place):
        if b >= 0:
            want_k[b], want_v[b] = pool.k[a], pool.v[a]
    assert torch.equal(k.cpu(), want_k) and torch.equal(v.cpu(), want_v)


@pytest.mark.parametrize("refs", [[0] * 9, [1] * 9, [0] * 8 + [2], [3] + [0] * 8, [0, 0, 0, 0, 1, 1, 1, 1, 1], [-1, 0, 1, -5, 2]])
def test_compact_small_pools(refs):
    k = torch.randn((len(refs), 2, 16, 64), device="cuda").bfloat16()
    was = k.clone()
    r = wb.cache_compact(wb.PagedCache(k, k.clone()), ints(refs))
    place, after, n = compacted(refs)
    assert (r.used.tolist(), r.place.tolist(), r.page_refs.tolist(), r.page_table, r.prefix_pages) == ([n], place, after, None, None)
    for a, b in enumerate(place):
        assert b < 0 or torch.equal(k[b], was[a])


@pytest.mark.parametrize("page, heads, dim, dtype, a, b, offset", [
    (16, 2, 64, torch.bfloat16, "hnd", "hnd", 0), (16, 2, 64, torch.bfloat16, "nhd", "nhd", 0), (64, 5, 128, torch.float16, "hnd", "nhd", 0),
    (64, 5, 128, torch.bfloat16, "nhd", "hnd", 0), (32, 3, 20, torch.bfloat16, "hnd", "nhd", 0), (16, 1, 2, torch.float16, "hnd", "hnd", 0),
    (16, 2, 64, torch.bfloat16, "hnd", "hnd", 1), (16, 2, 64, torch.bfloat16, "nhd", "hnd", 8), (1024, 2, 128, torch.bfloat16, "hnd", "nhd", 0)])
def test_copy(page, heads, dim, dtype, a, b, offset):
    g = torch.Generator().manual_seed(page + dim)

    def cache(n, order):
        x = torch.randn((n, page, heads, dim) if order == "nhd" else (n, heads, page, dim), generator=g).to(dtype)
        return x.transpose(1, 2) if order == "nhd" else x
    source, to = (cache(12, a), cache(12, a)), (cache(9, b), cache(9, b))
    src, dst = [on_gpu(x, offset) for x in source], [on_gpu(x, offset) for x in to]
    f, t = [3, 3, -1, 0, 11, 5], [8, 0, 2, -1, 4, 1]
    status = ints(NO_ERROR)
    wb.cache_copy(wb.PagedCache(*dst), ints(t), wb.PagedCache(*src), ints(f), dev_status=status)
    for x, s, d in zip(to, source, dst):
        want = x.clone()
        for i, j in zip(f, t):
            if i >= 0 and j >= 0:
                want[j] = s[i]
        assert torch.equal(d.cpu(), want)
    assert status.tolist() == NO_ERROR
    wb.cache_copy(wb.PagedCache(*dst), ints([]), wb.PagedCache(*src), ints([]))
    for f, t, want in (([0, 12], [1, 2], [89, 1, 12]), ([0, -2], [1, 2], [89, 1, -2]), ([0, 1, 2], [1, 2, 9], [90, 2, 9])):
        status.zero_()
        before = dst[0].clone()
        wb.cache_copy(wb.PagedCache(*dst), ints(t), wb.PagedCache(*src), ints(f), dev_status=status)
        assert status.tolist() == [wb.ERR_BAD_MASK] + want
        bad = {t[want[1]]}
        assert all(torch.equal(dst[0][j], before[j]) for j in range(9) if j not in t or j in bad)


def test_copy_inside_one_cache():
    k = torch.randn((20, 2, 16, 64), device="cuda").half()
    v = torch.randn((20, 2, 16, 64), device="cuda").half()
    wk, wv = k.clone(), v.clone()
    cache = wb.PagedCache(k, v)
    wb.cache_copy(cache, ints([1, 2, 3]), cache, ints([7, 7, 9]))
    wk[[1, 2, 3]], wv[[1, 2, 3]] = wk[[7, 7, 9]], wv[[7, 7, 9]]
    assert torch.equal(k, wk) and torch.equal(v, wv)


def test_pages_behind_two_to_the_31_elements():
    pages = 70000                                                      # of 32,768 elements: 4.6 GB a tensor
    k = torch.zeros((pages, 1, 256, 128), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    k[69000] = torch.randn((1, 256, 128), device="cuda")
    v[69000] = torch.randn((1, 256, 128), device="cuda")
    cache = wb.PagedCache(k, v)
    wb.cache_copy(cache, ints([69999]), cache, ints([69000]))
    assert torch.equal(k[69999], k[69000]) and torch.equal(v[69999], v[69000]) and k[69999].any()
    refs = torch.zeros((pages,), dtype=torch.int32, device="cuda")
    refs[69000] = 1
    table, new = wb.cache_fork(cache, ints([[69000]]), ints([200]), refs + (torch.arange(pages, device="cuda") < 69990).int(), ints([200, 200]), ints([200, 200]),
                               parents=ints([0, 0]), max_pages=1)
    assert table.tolist() == [[69990], [69991]]                         # (held from outside too)
    assert torch.equal(k[69991][:, :200], k[69000][:, :200]) and not k[69991][:, 200:].any()
    r = wb.cache_compact(cache, refs)
    assert r.used.tolist() == [1] and torch.equal(k[0], k[69000]) and torch.equal(v[0], v[69000])


def test_captured_steps_follow_their_tensors():
    pool = Pool(8, 200, seed=21, spare=6.0)
    k, v = on_gpu(pool.k), on_gpu(pool.v)
    cache = wb.PagedCache(k, v)
    table, held, refs = ints(pool.padded()), ints(pool.held), ints(pool.refs)
    keep, room, parents = ints([0] * 8), ints([0] * 8), ints([-1] * 8)
    out, refs_out = ints([[0] * 40] * 8), torch.empty_like(refs)
    workspace = torch.empty((1 << 20,), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call = lambda **kw: wb.cache_fork(cache, table, held, refs, keep, room, parents=parents, table_out=out, refs_out=refs_out, workspace=workspace, **kw)  # noqa: E731
    with torch.cuda.stream(side):
        call()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            call()
            compact = wb.cache_compact(cache, refs_out, page_table=out, workspace=workspace)
    torch.cuda.synchronize()
    for seed in range(3):
        parent, n, m = wishes(pool, 8, seed)
        for t, x in ((parents, parent), (keep, n), (room, m)):
            t.copy_(ints(x))
        k.copy_(pool.k), v.copy_(pool.v)
        graph.replay()
        torch.cuda.synchronize()
        rows, counts, copies = forked(pool.table, pool.held, pool.refs, n, m, parent, 16)
        assert out.tolist() == [r + [-1] * (40 - len(r)) for r in rows] and refs_out.tolist() == counts
        place, _, used = compacted(counts)
        assert compact.used.tolist() == [used] and compact.page_table.tolist() == [[place[p] for p in r] + [-1] * (40 - len(r)) for r in rows]


def test_calls_on_two_streams():
    pools = [Pool(200, 900, seed=30 + i, spare=3.0, heads=1) for i in range(2)]
    jobs = []
    for i, pool in enumerate(pools):
        parents, keep, room = wishes(pool, 150, i)
        args = [ints(pool.padded()), ints(pool.held), ints(pool.refs), ints(keep), ints(room)]
        jobs.append((pool, parents, keep, room, wb.PagedCache(on_gpu(pool.k), on_gpu(pool.v)), args, ints(parents), torch.cuda.Stream()))
    torch.cuda.synchronize()
    results = [[wb.cache_fork(cache, *args, parents=parent, stream=stream) for _, _, _, _, cache, args, parent, stream in jobs] for _ in range(5)]
    torch.cuda.synchronize()
    for i, (pool, parents, keep, room, *_rest) in enumerate(jobs):
        rows, counts, _ = forked(pool.table, pool.held, pool.refs, keep, room, parents, 16)
        for turn in results:
            table, refs = turn[i]
            assert refs.tolist() == counts and table.tolist() == [r + [-1] * (table.shape[1] - len(r)) for r in rows]
