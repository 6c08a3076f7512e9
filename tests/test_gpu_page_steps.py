"""Forks and compactions as a program meets them beyond test_gpu_pages.py, against the same definitions on lists."""
import random

import pytest
import torch

from paper_2609_34814_b200 import binding as wb
from pages_util import Pool, forked, ints, on_gpu, up
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
