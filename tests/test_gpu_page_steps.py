"""Forks and compactions as a program meets them beyond test_gpu_pages.py, against the same definitions on lists."""
import os
import random
import subprocess
import sys

import pytest
import torch

from paper_2609_34814_b200 import binding as wb
from pages_util import Pool, forked, ints, on_gpu
from test_gpu_pages import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("old_rows, tokens, rows", [(1, 1000, 64), (2, 2500, 130), (1, 16000, 66), (1, 16000, 280), (2, 30000, 900)])
def test_few_rows_go_on_in_many_ways_of_different_lengths(old_rows, tokens, rows):
    """The new rows' entries are most of the work, however small the pool and the last table are."""
    pool = Pool(old_rows, tokens, page=16, heads=1, dim=2, shared=0.0, spare=2.0 * rows * 16 / tokens + 1.0, seed=rows)
    r = random.Random(rows)
    parents = [b % old_rows for b in range(rows)]
    keep = [r.randint(0, pool.held[p]) for p in parents]
    check(pool, parents, keep, [n + r.choice([0, 1, 16]) for n in keep])


@pytest.mark.parametrize("stream", [False, True])
def test_results_are_tensors_of_their_own(stream):
    """A result that is kept or saved holds its own numbers and nothing else: no other result, no workspace."""
    kw = dict(stream=torch.cuda.Stream()) if stream else {}
    pool = Pool(6, 300, seed=33, spare=3.0)
    cache, held = wb.PagedCache(on_gpu(pool.k), on_gpu(pool.v)), ints(pool.held)
    table, refs, prefix = ints(pool.padded()), ints(pool.refs), ints(pool.prefix)
    torch.cuda.synchronize()
    results = [*wb.cache_fork(cache, table, held, refs, held, held, **kw)]
    torch.cuda.synchronize()
    results += wb.cache_compact(cache, results[1], page_table=results[0], prefix_pages=prefix, **kw)
    x = torch.randn((2, 300, 64), device="cuda").bfloat16()
    torch.cuda.synchronize()
    results += wb.prompt_attn(x, x, x, ints([0, 100, 300]), return_lse=True, **kw)
    torch.cuda.synchronize()
    assert len({t.untyped_storage().data_ptr() for t in results}) == len(results) == 9
    for t in results:
        assert t.untyped_storage().nbytes() == t.numel() * t.element_size() and not t._is_view()


def test_what_a_fork_that_runs_out_of_pages_leaves():
    """Rows in front of the first that is short have everything, pages written may be such as ended rows have let go of, and the new table goes on."""
    pool = Pool(4, 40, page=16, spare=0.0, seed=34, shared=0.0, outside=0.0)
    pool.held = [40, 20, 16, 8]
    pool.table, pool.wide = [[5, 2, 7], [0, 9], [4], [1]], 3
    pool.n_pages = 10
    pool.refs = [1, 1, 1, 0, 1, 1, 0, 1, 0, 1]
    shape = (10,) + tuple(pool.k.shape[1:])
    pool.k, pool.v = (torch.randn(shape).bfloat16() for _ in range(2))
    k, v = on_gpu(pool.k), on_gpu(pool.v)
    cache, status = wb.PagedCache(k, v), ints([0] * 4)
    # rows 1 and 3 end, row 0 goes on in four ways with copies of page 7: pages 0, 1, 3, 6, 8, 9 are free
    parents, keep, room = [0, 0, 2, 0, 0, 2], [40, 40, 16, 40, 40, 16], [49, 49, 16, 48, 64, 40]
    table, refs = wb.cache_fork(cache, ints(pool.padded()), ints(pool.held), ints(pool.refs), ints(keep), ints(room), parents=ints(parents), max_pages=5,
                                dev_status=status)
    rows, counts, copies = forked(pool.table, pool.held, pool.refs, keep, room, parents, 16)
    assert table.tolist() == [r + [-1] * (5 - len(r)) for r in rows] and refs.tolist() == counts
    assert table.tolist() == [[5, 2, 7, 0, -1], [5, 2, 1, 3, -1], [4, -1, -1, -1, -1], [5, 2, 6, -1, -1], [5, 2, 8, 9, -1], [4, -1, -1, -1, -1]]
    assert status.tolist() == [wb.ERR_NO_PAGES, 85, 5, 2]
    want_k, want_v = pool.k.clone(), pool.v.clone()
    for a, b, n in copies:
        want_k[b, :, :n], want_v[b, :, :n] = pool.k[a, :, :n], pool.v[a, :, :n]
    assert torch.equal(k.cpu(), want_k) and torch.equal(v.cpu(), want_v)
    assert {b for _, b, _ in copies} == {1, 6, 8} and not torch.equal(k[1].cpu(), pool.k[1])     # page 1 was row 3's
    # without the last row, and nobody short
    status.zero_()
    table, refs = wb.cache_fork(cache, table, ints([49, 49, 16, 48, 64, 16]), refs, ints([49, 16, 48]), ints([49, 16, 60]), parents=ints([0, 2, 3]), dev_status=status)
    assert status.tolist() == [0] * 4 and table.tolist() == [[5, 2, 7, 0, -1], [4, -1, -1, -1, -1], [5, 2, 6, 1, -1]]


FIRST = """
import torch
from paper_2609_34814_b200 import binding as wb

pages, rows = 400000, 512
ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
cache = wb.PagedCache(*(torch.zeros((pages, 1, 16, 8), dtype=torch.bfloat16, device="cuda") for _ in range(2)))
refs, table, held = torch.zeros(pages, dtype=torch.int32, device="cuda"), ints([[-1] * 4] * rows), ints([0] * rows)
keep, room = ints([0] * rows), ints([40] * rows)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    new, counts = wb.cache_fork(cache, table, held, refs, keep, room)
    r = wb.cache_compact(cache, counts, page_table=new)
graph.replay()
torch.cuda.synchronize()
assert new.tolist() == [[3 * b, 3 * b + 1, 3 * b + 2, -1] for b in range(rows)]
assert r.used.item() == 3 * rows and torch.equal(r.page_table, new)
print("captured")
"""


def test_the_first_call_of_a_program_may_be_captured():
    """What the largest clusters have to be asked for is asked for in that call."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", FIRST], cwd=root, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and "captured" in done.stdout, done.stderr[-2000:]
