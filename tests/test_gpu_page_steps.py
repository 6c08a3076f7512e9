"""Forks and compactions as a program meets them beyond test_gpu_pages.py, against the same definitions on lists."""
import os
import random
import subprocess
import sys

import pytest
import torch

from paper_2609_34814_b200 import binding as wb
from pages_util import Pool, ints, on_gpu
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
