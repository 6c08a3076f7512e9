"""Attention over a shared prefix and each sequence's own keys, against the definition in 64 bits."""
import copy
import math

import pytest
import torch

from paper_2609_34814_b200 import binding as wb
from tests.serving_util import Batch

BF16, FP16 = torch.bfloat16, torch.float16


def call(b, causal=True, **kw):
    cache = wb.PagedCache(b.k, b.v)
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    o, lse = wb.prefix_attn(cache, b.q, b.seq_start, b.kv_len, b.table if b.table.shape[1] else None,
                            b.prefix_pages if b.prefix else None, b.prefix, causal=causal, return_lse=True, dev_status=status, **kw)
    return o, lse, status


def check(b, causal=True, scale=None, expect_status=True):
    o, lse, o_tol, lse_tol = b.expected(causal, scale)
    b.cuda()
    got, got_lse, status = call(b, causal, **({} if scale is None else {"scale": scale}))
    torch.cuda.synchronize()
    assert status.tolist() == [0, 0, 0, 0]
    live = sum(b.new)
    off = (got.double().cpu() - o)[:, :live].abs()
    assert bool((off <= o_tol[:, :live]).all()), float((off - o_tol[:, :live]).max())
    got_lse = got_lse.double().cpu()[:, :live]
    empty = lse[:, :live] == -math.inf
    assert torch.equal(got_lse == -math.inf, empty)
    assert bool(((got_lse - lse[:, :live]).abs()[~empty] <= lse_tol[:, :live][~empty]).all())
    assert bool((got[:, :live].cpu()[empty] == 0).all())


CASES = {
    "one_token_one_key": dict(new=[1], own=[1], prefix=0),
    "one_token_prefix_only": dict(new=[1], own=[0], prefix=1, causal=False),
    "prefix_of_one_and_own_of_one": dict(new=[1, 1], own=[1, 1], prefix=1, group=4),
    "tile_edges": dict(new=[1] * 6, own=[127, 128, 129, 255, 256, 257], prefix=128, group=4),
    "prefix_edges_127": dict(new=[1, 2], own=[3, 2], prefix=127, group=8),
    "prefix_edges_129": dict(new=[1, 2], own=[3, 2], prefix=129, group=8),
    "odd_group_5": dict(new=[1, 3, 30], own=[40, 3, 31], prefix=300, group=5, page=32),
    "odd_group_7_dim64": dict(new=[2, 1, 19], own=[70, 130, 19], prefix=200, group=7, dim=64, page=64, dtype=FP16, token_major=True),
    "group_128": dict(new=[1, 3], own=[20, 140], prefix=150, kv_heads=1, group=128, page=16),
    "group_65_leaves_half_the_rows": dict(new=[2, 3], own=[20, 140], prefix=50, kv_heads=1, group=65, dim=64),
    "more_than_one_row_tile": dict(new=[100, 70, 1], own=[150, 70, 400], prefix=260, group=2, page=128),
    "more_than_two_row_tiles": dict(new=[300, 7], own=[300, 300], prefix=140, group=1, page=64, kv_heads=1),
    "own_only": dict(new=[1, 40, 300], own=[513, 40, 700], prefix=0, kv_heads=1, page=256, dim=64),
    "full_own": dict(new=[5, 140], own=[300, 141], prefix=77, group=2, causal=False, page=128),
    "no_new_tokens_in_some": dict(new=[0, 1, 0, 2, 0], own=[10, 20, 0, 2, 500], prefix=40, group=4),
    "rows_that_see_nothing": dict(new=[5, 1], own=[2, 1], prefix=0, group=3),
    "fewer_keys_than_new_tokens": dict(new=[6, 130], own=[2, 100], prefix=33, group=2),
    "no_own_keys": dict(new=[1, 4], own=[0, 0], prefix=333, group=4, causal=False),
    "tokens_of_no_sequence": dict(new=[3, 2], own=[9, 200], prefix=64, group=2, spare_tokens=5),
    "fp16_dim128": dict(new=[1, 1, 1], own=[1, 200, 900], prefix=1000, group=4, dtype=FP16),
    "token_major_small_pages": dict(new=[1, 9], own=[30, 65], prefix=210, group=4, token_major=True),
    "page_larger_than_a_tile": dict(new=[1, 3], own=[700, 600], prefix=900, group=2, page=512),
    "many_parts": dict(new=[1, 1], own=[4000, 10], prefix=20000, kv_heads=1, group=2, page=64),
    "rising_scores": dict(new=[1, 50], own=[300, 600], prefix=700, group=2, rise=12.0, q_scale=4.0),
    "nearly_one_hot": dict(new=[1, 2], own=[300, 200], prefix=300, group=4, q_scale=20.0, dim=64),
}


@pytest.mark.gpu
@pytest.mark.parametrize("name", CASES)
def test_matches_definition(name):
    c = dict(CASES[name])
    causal = c.pop("causal", True)
    check(Batch(**c, seed=len(name)), causal)


@pytest.mark.gpu
def test_batch_larger_than_a_block():
    n = 900
    check(Batch(new=[i % 3 for i in range(n)], own=[3 + i % 41 for i in range(n)], prefix=50, kv_heads=1, group=2, dim=64))


@pytest.mark.gpu
def test_scale_is_used():
    check(Batch(new=[1, 3], own=[30, 40], prefix=100, group=2), scale=0.3)


@pytest.mark.gpu
def test_more_prefix_units_than_ctas():
    # 160 key heads with one unit each: 148 go whole, the others are cut up; compared with calls of a head each
    b = Batch(new=[2, 1, 1], own=[10, 20, 300], prefix=300, kv_heads=160, group=1, dim=64, seed=3).cuda()
    o, lse, status = call(b)
    assert status.tolist() == [0] * 4
    for h in (0, 77, 147, 148, 159):
        one = wb.PagedCache(b.k[:, h:h + 1], b.v[:, h:h + 1])
        oh, lh = wb.prefix_attn(one, b.q[h:h + 1], b.seq_start, b.kv_len, b.table, b.prefix_pages, b.prefix, return_lse=True)
        assert float((oh.float() - o[h:h + 1].float()).abs().max()) <= 2.0 ** -7 * float(o[h].abs().max())
        assert float((lh - lse[h:h + 1]).abs().max()) <= 1e-5


@pytest.mark.gpu
def test_same_bits_every_time_and_untouched_tokens():
    b = Batch(new=[1, 30, 1], own=[500, 90, 7], prefix=3000, group=4, spare_tokens=4, seed=5).cuda()
    o = torch.full((b.tokens, b.heads, b.dim), 7.0, dtype=b.dtype, device="cuda").transpose(0, 1)
    first, lse, _ = call(b, o=o)
    live = sum(b.new)
    assert bool((first[:, live:] == 7).all())
    first = first.clone()
    for _ in range(20):
        again, lse2, _ = call(b)
        assert torch.equal(again[:, :live], first[:, :live]) and torch.equal(lse2[:, :live], lse[:, :live])


@pytest.mark.gpu
@pytest.mark.parametrize("new,own,group,prefix", [
    # rows that leave warps without any (16 x 5 = 80, 33, 3 x 11 = 33 of 128), keys that end in a first half tile, many short items one behind the other
    (26, [26 + 37 * i % 290 for i in range(83)], 8, 2),
    (5, [5 + 61 * i % 190 for i in range(300)], 16, 0),
    (33, [33 + 29 * i % 100 for i in range(150)], 1, 20),
    (11, [11, 64, 65, 128, 129, 192, 40, 200] * 30, 3, 0),
])
def test_warps_without_rows_do_not_run_ahead(new, own, group, prefix):
    b = Batch(new=[new] * len(own), own=own, prefix=prefix, kv_heads=4, group=group, page=256, dtype=FP16, seed=len(own))
    check(b)
    first, lse, _ = call(b)
    first, lse = first.clone(), lse.clone()
    for _ in range(20):
        again, lse2, _ = call(b)
        assert torch.equal(again, first) and torch.equal(lse2, lse)


@pytest.mark.gpu
def test_strides_of_q_and_o():
    b = Batch(new=[2, 5], own=[40, 60], prefix=130, group=2, seed=6)
    o, lse, o_tol, _ = b.expected(True)
    b.cuda()
    wide = torch.zeros((b.heads + 3, b.tokens + 2, b.dim + 64), dtype=b.dtype, device="cuda")
    q = wide[1:1 + b.heads, 1:1 + b.tokens, 8:8 + b.dim]
    q.copy_(b.q)
    b.q = q
    out = torch.zeros((b.heads, b.tokens, 3 * b.dim), dtype=b.dtype, device="cuda")[..., b.dim:2 * b.dim]
    got, _, _ = call(b, o=out)
    assert bool(((got.double().cpu() - o).abs() <= o_tol).all())


@pytest.mark.gpu
def test_lengths_change_under_a_captured_call():
    b = Batch(new=[1, 1, 1], own=[300, 40, 90], prefix=500, group=4, seed=7)
    c = Batch(new=[1, 1, 1], own=[300, 40, 90], prefix=500, group=4, seed=7)
    c.own = [17, 1, 64]
    c.kv_len = torch.tensor(c.own, dtype=torch.int32)
    want = [x.expected(True) for x in (b, c)]
    lens = [b.kv_len.cuda(), c.kv_len.cuda()]
    b.cuda()
    cache = wb.PagedCache(b.k, b.v)
    o, lse = torch.empty_like(b.q), torch.empty((b.heads, b.tokens), dtype=torch.float32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ws = wb.prefix_attn_workspace_bytes(cache, wb.batch_desc(b.heads, b.tokens, b.seq_start, b.kv_len, b.table, b.prefix))
        ws = torch.empty((ws,), dtype=torch.uint8, device="cuda")
        run = lambda: wb.prefix_attn(cache, b.q, b.seq_start, b.kv_len, b.table, b.prefix_pages, b.prefix, o=o, lse=lse, workspace=ws)  # noqa: E731
        run()
        assert wb.last_launch_count() == 2
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            run()
    torch.cuda.synchronize()
    for n, (eo, el, eo_tol, el_tol) in zip(lens, want):
        b.kv_len.copy_(n)
        graph.replay()
        torch.cuda.synchronize()
        assert bool(((o.double().cpu() - eo).abs() <= eo_tol).all())
        assert bool(((lse.double().cpu() - el).abs() <= el_tol).all())


@pytest.mark.gpu
def test_other_stream():
    b = Batch(new=[1, 1], own=[300, 40], prefix=500, group=4, seed=8)
    o, _, o_tol, _ = b.expected(True)
    b.cuda()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    out = torch.empty_like(b.q)
    cache = wb.PagedCache(b.k, b.v)
    ws = torch.empty((wb.prefix_attn_workspace_bytes(cache, wb.batch_desc(b.heads, b.tokens, b.seq_start, b.kv_len, b.table, b.prefix)),),
                     dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    wb.prefix_attn(cache, b.q, b.seq_start, b.kv_len, b.table, b.prefix_pages, b.prefix, o=out, workspace=ws, stream=side)
    side.synchronize()
    assert bool(((out.double().cpu() - o).abs() <= o_tol).all())


@pytest.mark.gpu
def test_workspace_of_another_stream_is_not_handed_on():
    b = Batch(new=[1, 1], own=[300, 40], prefix=500, group=4, seed=8)
    o, _, o_tol, _ = b.expected(True)
    b.cuda()
    cache = wb.PagedCache(b.k, b.v)
    size = wb.prefix_attn_workspace_bytes(cache, wb.batch_desc(b.heads, b.tokens, b.seq_start, b.kv_len, b.table, b.prefix))
    side, busy = torch.cuda.Stream(), torch.randn((4096, 4096), device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            busy @ busy                                  # some ms in front of the call
    got, lse = wb.prefix_attn(cache, b.q, b.seq_start, b.kv_len, b.table, b.prefix_pages, b.prefix, return_lse=True, stream=side)
    for _ in range(8):                                   # the current stream takes memory of the workspace's size and writes to it
        torch.empty((size,), dtype=torch.uint8, device="cuda").fill_(255)
    side.synchronize()
    torch.cuda.synchronize()
    assert bool(((got.double().cpu() - o).abs() <= o_tol).all())


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    # pages of 65,536 slots, 8 heads of 64: 2^25 elements each, 72 pages = 2.4e9 elements; the keys lie in the last ones
    page, heads, dim, n = 65536, 8, 64, 72
    k = torch.zeros((n, heads, page, dim), dtype=BF16, device="cuda")
    v = torch.zeros((n, heads, page, dim), dtype=BF16, device="cuda")
    small = Batch(new=[1, 2], own=[200, 90], prefix=300, kv_heads=heads, group=1, dim=dim, page=65536 // 128, seed=9)
    o, lse, o_tol, lse_tol = small.expected(True)
    places = {"prefix": n - 1, 0: n - 2, 1: n - 3}
    for name, keys, pages in [("prefix", 300, small.prefix_pages), (0, 200, small.table[0]), (1, 90, small.table[1])]:
        k[places[name], :, :keys] = small.get(small.k, pages, keys).to(BF16).cuda()
        v[places[name], :, :keys] = small.get(small.v, pages, keys).to(BF16).cuda()
    small.cuda()
    table = torch.tensor([[n - 2], [n - 3]], dtype=torch.int32, device="cuda")
    got, got_lse = wb.prefix_attn(wb.PagedCache(k, v), small.q, small.seq_start, small.kv_len, table,
                                  torch.tensor([n - 1], dtype=torch.int32, device="cuda"), 300, return_lse=True)
    assert bool(((got.double().cpu() - o).abs() <= o_tol).all())
    assert bool(((got_lse.double().cpu() - lse).abs() <= lse_tol).all())


@pytest.mark.gpu
def test_malformed_is_reported_and_the_rest_is_right():
    def fresh():
        return Batch(new=[1, 1, 1], own=[100, 50, 70], prefix=64, group=2, seed=10)
    good = fresh()
    o, _, o_tol, _ = good.expected(True)
    for what, code in (("len", 51), ("negative len", 51), ("start", 50), ("page", 52), ("prefix page", 52)):
        b = fresh().cuda()
        if what == "len":
            b.kv_len[1] = b.table.shape[1] * b.page + 1
        elif what == "negative len":
            b.kv_len[1] = -1
        elif what == "start":
            b.seq_start[3] = b.tokens + 9
        elif what == "page":
            b.table[1, 1] = b.n_pages
        else:
            b.prefix_pages[0] = -1
        got, _, status = call(b)
        status = status.tolist()
        assert status[0] == wb.ERR_BAD_MASK and status[1] == code, (what, status)
        if what == "start":
            assert status[2:] == [2, b.tokens + 9]
        elif what != "prefix page":
            assert status[2] == 1
        if what != "prefix page":
            keep = [0, 1] if what == "start" else [0, 2]
            assert bool(((got.double().cpu() - o).abs() <= o_tol)[:, keep].all()), what


# starts that decrease: (starts, lens, sequences whose outputs are right, whom the status may name with which value)
DECREASING = {
    "overlaps_the_first": ([0, 10, 5, 8], [60, 20, 300], [0], [(1, 5)]),
    "and_goes_on_behind_it": ([0, 10, 5, 8, 13, 16], [700, 20, 30, 90, 40], [0, 4], [(1, 5)]),
    "a_start_out_of_range_between": ([0, 10, -1, 5, 13, 16], [50, 20, 30, 90, 40], [0, 4], [(1, -1), (2, -1)]),
    "too_large_in_front_of_the_others": ([0, 100, 4, 9, 16], [40, 20, 200, 70], [2, 3], [(0, 100), (1, 4)]),
    "from_behind": ([9, 3, 9, 16], [40, 70, 200], [2], [(0, 3)]),
    "many": (list(range(451)) + list(range(100, 1000)), [1 + i % 90 for i in range(1350)], [i for i in range(1350) if i < 450 or i >= 801], [(450, 100)]),
}


@pytest.mark.gpu
@pytest.mark.parametrize("prefix", [0, 200])
@pytest.mark.parametrize("name", DECREASING)
def test_a_start_that_decreases_spoils_no_other_sequence(name, prefix):
    starts, own, right, named = DECREASING[name]
    new = [starts[b + 1] - starts[b] if b in set(right) else 0 for b in range(len(own))]
    live = [t for b in right for t in range(starts[b], starts[b + 1])]
    tokens = min(max(starts), 2000) if name != "too_large_in_front_of_the_others" else 16
    own = [max(n, k) for n, k in zip(new, own)]
    b = Batch(new=new, own=own, prefix=prefix, group=2 if len(own) < 20 else 1, dim=64, seed=13, spare_tokens=tokens - sum(new))
    b.seq_start = torch.tensor(starts, dtype=torch.int32)
    o, lse, o_tol, lse_tol = b.expected(True)
    b.cuda()
    out = torch.full((b.tokens, b.heads, b.dim), 7.0, dtype=b.dtype, device="cuda").transpose(0, 1)
    got, got_lse, status = call(b, o=out)
    assert status.tolist() in [[wb.ERR_BAD_MASK, 50, *x] for x in named]
    assert bool(((got.double().cpu() - o).abs() <= o_tol)[:, live].all())
    assert bool(((got_lse.double().cpu() - lse).abs() <= lse_tol)[:, live].all())
    others = [t for t in range(tokens) if t not in set(live)]
    assert bool((got[:, others] == 7).all())                      # tokens of no sequence are left alone


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [True, False])
def test_wide_prefix_units_dealt_whole(causal):
    # 80 key heads of three units over six key tiles: 148 of the 240 go whole, head 49's second one begins the line
    b = Batch(new=[300, 200, 100], own=[310, 200, 350], prefix=700, kv_heads=80, group=1, dim=64, page=64, seed=14)
    some = [0, 48, 49, 50, 79]
    few = copy.copy(b)
    few.k, few.v, few.q, few.kv_heads, few.heads = b.k[:, some], b.v[:, some], b.q[some], len(some), len(some)
    o, lse, o_tol, lse_tol = few.expected(causal)
    b.cuda()
    got, got_lse, status = call(b, causal)
    assert status.tolist() == [0] * 4
    assert bool(((got[some].double().cpu() - o).abs() <= o_tol).all())
    assert bool(((got_lse[some].double().cpu() - lse).abs() <= lse_tol).all())


@pytest.mark.gpu
@pytest.mark.parametrize("new, own, prefix, group, dim", [
    (1, 5, 0, 2, 128), (1, 40, 300, 4, 64), (3, 200, 0, 4, 128),          # few rows
    (20, 90, 0, 4, 64), (20, 30, 500, 3, 128),                            # narrow
    (150, 400, 0, 1, 128), (150, 200, 300, 2, 64),                        # wide
])
def test_infinite_and_nan_scores(new, own, prefix, group, dim):
    # one key of each list holds +infinity in one channel: a row's score there is +infinity or -infinity by its query's sign, and with
    # -infinity the row is as if the key were not there; one row's query is NaN
    b = Batch(new=[new, new], own=[own, own], prefix=prefix, kv_heads=2, group=group, dim=dim, page=32, seed=15)
    hit = [(b.table[0], 1)] + ([(b.prefix_pages, prefix // 2)] if prefix else [])      # keys that every new token of sequence 0 sees
    for pages, key in hit:
        b.k[int(pages[key // b.page]), :, key % b.page, 3] = math.inf
    b.q[:, new - 1, 7] = math.nan                                 # sequence 0's last token
    finite = copy.copy(b)
    finite.prefix, finite.own = max(prefix - 1, 0), [own - 1, own]

    def get(cache, pages, n):
        for where, key in hit:
            if torch.equal(pages, where):
                x = b.get(cache, pages, n + 1)
                return torch.cat([x[:, :key], x[:, key + 1:]], 1)
        return b.get(cache, pages, n)
    finite.get = get
    o, lse, o_tol, lse_tol = finite.expected(True)
    sees = torch.zeros((b.heads, b.tokens), dtype=torch.bool)      # tokens with a key that holds the infinity in sight
    sees[:, :new] = True
    if prefix:
        sees[:] = True
    q3 = b.q[..., 3].double()
    nan = (sees & (q3 >= 0)) | b.q.isnan().any(-1)
    b.cuda()
    got, got_lse, status = call(b)
    assert status.tolist() == [0] * 4
    got, got_lse = got.double().cpu(), got_lse.double().cpu()
    assert bool(got[nan].isnan().all()) and bool(got_lse[nan].isnan().all())
    assert bool(((got - o).abs() <= o_tol)[~nan].all()) and bool(((got_lse - lse).abs() <= lse_tol)[~nan].all())
    assert bool(nan.any()) and bool((~nan).any())


@pytest.mark.gpu
@pytest.mark.parametrize("new, group", [(1, 2), (20, 4), (150, 1)])
def test_scores_that_are_all_minus_infinity_count_as_none(new, group):
    b = Batch(new=[new], own=[new], prefix=0, group=group, dim=64, seed=16)
    b.k[..., 2] = torch.where(b.k[..., 2].isnan(), b.k[..., 2], torch.full_like(b.k[..., 2], -math.inf))
    b.q[..., 2] = 1.0
    b.cuda()
    got, lse, status = call(b)
    assert status.tolist() == [0] * 4
    assert bool((got == 0).all()) and bool((lse == -math.inf).all())


@pytest.mark.gpu
def test_a_wait_that_runs_out_leaves_the_context_usable():
    b = Batch(new=[1, 1], own=[300, 40], prefix=500, group=4, seed=11)
    o, _, o_tol, _ = b.expected(True)
    b.cuda()
    _, _, status = call(b, flags=wb.PREFIX_SELFTEST_LOST_TILE)
    torch.cuda.synchronize()
    assert status[0].item() == wb.ERR_TIMEOUT
    got, _, status = call(b)
    assert status.tolist() == [0] * 4
    assert bool(((got.double().cpu() - o).abs() <= o_tol).all())


@pytest.mark.gpu
@pytest.mark.parametrize("fill", [0x00, 0x7f, 0xff])
@pytest.mark.parametrize("shape", [
    dict(new=[1] * 900, own=[5] * 900, prefix=0, kv_heads=8, group=2),            # ~48 own units of block 0, eight of them planned before it gives up
    dict(new=[2, 1, 1], own=[10, 20, 300], prefix=300, kv_heads=160, group=1),    # a whole prefix unit, then some that are cut
])
def test_a_wait_that_runs_out_with_units_never_planned(shape, fill):
    # what the workspace held before must not be taken for places of parts
    b = Batch(**shape, dim=64, seed=12).cuda()
    cache = wb.PagedCache(b.k, b.v)
    ws = torch.empty((wb.prefix_attn_workspace_bytes(cache, wb.batch_desc(b.heads, b.tokens, b.seq_start, b.kv_len, b.table, b.prefix)),),
                     dtype=torch.uint8, device="cuda")
    want, want_lse, _ = call(b, workspace=ws)
    want, want_lse = want.clone(), want_lse.clone()
    ws.fill_(fill)
    _, _, status = call(b, workspace=ws, flags=wb.PREFIX_SELFTEST_LOST_TILE)
    torch.cuda.synchronize()
    assert status[0].item() == wb.ERR_TIMEOUT
    got, got_lse, status = call(b, workspace=ws)
    assert status.tolist() == [0] * 4
    assert torch.equal(got, want) and torch.equal(got_lse, want_lse)


@pytest.mark.gpu
def test_tensors_the_kernels_must_not_write_to_are_refused():
    b = Batch(new=[1, 1], own=[300, 40], prefix=500, group=4, seed=17).cuda()
    cache = wb.PagedCache(b.k, b.v)
    size = wb.prefix_attn_workspace_bytes(cache, wb.batch_desc(b.heads, b.tokens, b.seq_start, b.kv_len, b.table, b.prefix))
    attend = lambda **kw: wb.prefix_attn(cache, b.q, b.seq_start, b.kv_len, b.table, b.prefix_pages, b.prefix, **kw)  # noqa: E731
    append = lambda **kw: wb.cache_append(cache, b.k[0, :, :2], b.v[0, :, :2], b.seq_start, b.kv_len, b.table, **kw)  # noqa: E731
    kept = b.k.clone()
    for bad in (dict(lse=torch.empty((b.heads, b.tokens))), dict(workspace=torch.empty((size,), dtype=torch.uint8)),
                dict(workspace=torch.empty((1,), dtype=torch.uint8, device="cuda").expand(size)),
                dict(workspace=torch.empty((size // 4,), dtype=torch.float32, device="cuda"))):
        with pytest.raises((TypeError, ValueError)):
            attend(**bad)
    for bad in (torch.zeros(4, dtype=torch.int32), torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda"),
                torch.zeros(1, dtype=torch.int32, device="cuda").expand(4), torch.zeros(8, dtype=torch.int32, device="cuda")[::2]):
        for run in (attend, append):
            with pytest.raises((TypeError, ValueError)):
                run(dev_status=bad)
    assert torch.equal(b.k.view(torch.int16), kept.view(torch.int16))


@pytest.mark.gpu
def test_empty_calls():
    b = Batch(new=[0, 0], own=[5, 6], prefix=30, group=2).cuda()
    o, lse, status = call(b)
    assert o.shape[1] == 0 and wb.last_launch_count() == 0 and status.tolist() == [0] * 4
