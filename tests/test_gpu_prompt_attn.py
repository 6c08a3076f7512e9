"""Attention of whole prompts against the definition in 64 bits.

What a result may be off: a score is a sum of head_dim products in fp32 and is scaled (head_dim + 2 roundings of partial sums that are at most
|q|.|k|), its exponential is good to 2^-20, the probability is rounded to the tensors' type (half a step: UNIT) before the second product,
whose sum is fp32, and the result is rounded once more.  So with e = (head_dim + 2) 2^-24 scale max |q|.|k| + 2^-20
    |lse error| <= e + 2^-22 |lse|,   |o error| <= (UNIT + 2 e) sum p |v| + UNIT |o| + 2^-24.
fp16 has a smallest step, 2^-24: below 2^-14 a probability is off by up to half of that and not by UNIT of itself.  Probabilities are taken relative to a
reference that is no more than the row's largest score, so their sum is at least 1 and |o error| is up to 2^-25 sum |v| more, over the keys that the row
sees.  (The sum itself is taken before the rounding.)  In bf16 the smallest step is 2^-133."""
import math

import pytest
import torch

from paper_2609_34814_b200 import binding as wb
from serving_util import UNIT

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


def tensors(tokens, heads, kv_heads, dim, dtype, order="nhd", seed=0, q_scale=1.0, ramp=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def one(h, scale=1.0):
        x = torch.randn((h, tokens, dim) if order == "hnd" else (tokens, h, dim), generator=g, device="cuda") * scale
        return x.to(dtype) if order == "hnd" else x.to(dtype).transpose(0, 1)
    q, k, v = one(heads, q_scale), one(kv_heads), one(kv_heads)
    if ramp:
        k = (k.float() * (1.0 + ramp * torch.arange(tokens, device="cuda")[:, None] / tokens)).to(dtype)
    return q, k, v


def expected(q, k, v, starts, lens, causal, scale=None):
    """o, lse, their tolerances; NaN where no sequence has a token"""
    heads, tokens, dim = q.shape
    group = heads // k.shape[0]
    scale = scale or 1.0 / math.sqrt(dim)
    unit = UNIT[q.dtype]
    o = torch.full(q.shape, math.nan, dtype=torch.float64, device="cuda")
    lse = torch.full(q.shape[:2], math.nan, dtype=torch.float64, device="cuda")
    o_tol, lse_tol = torch.zeros_like(o), torch.zeros_like(lse)
    for s, n in zip(starts, lens):
        if n == 0:
            continue
        at = slice(s, s + n)
        for h in range(heads):
            qh, kh, vh = q[h, at].double(), k[h // group, at].double(), v[h // group, at].double()
            x = qh @ kh.t() * scale
            size = qh.abs() @ kh.abs().t() * scale
            if causal:
                hidden = torch.ones((n, n), dtype=torch.bool, device="cuda").triu(1)
                x, size = x.masked_fill(hidden, -math.inf), size.masked_fill(hidden, 0.0)
            w = torch.softmax(x, -1)
            o[h, at], lse[h, at] = w @ vh, torch.logsumexp(x, -1)
            e = (dim + 2) * 2.0 ** -24 * size.amax(-1) + 2.0 ** -20
            lse_tol[h, at] = e + 2.0 ** -22 * lse[h, at].abs()
            o_tol[h, at] = (w @ vh.abs()) * (unit + 2 * e)[:, None] + o[h, at].abs() * unit + 2.0 ** -24
            if q.dtype == HF:
                o_tol[h, at] += 2.0 ** -25 * (vh.abs().cumsum(0) if causal else vh.abs().sum(0))
    return o, lse, o_tol, lse_tol


def run(q, k, v, starts, lens=None, **kw):
    """(o, lse, status); outputs are filled with 7 before the call"""
    seq_start = torch.tensor(starts, dtype=torch.int32, device="cuda")
    seq_len = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    o, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    wb.prompt_attn(q, k, v, seq_start, seq_len=seq_len, o=o, lse=lse, dev_status=status, **kw)
    return o, lse, status.tolist()


def check(q, k, v, starts, lens=None, causal=True, scale=0.0):
    o, lse, status = run(q, k, v, starts, lens, causal=causal, scale=scale)
    assert status == [0, 0, 0, 0]
    n = [b - a for a, b in zip(starts, starts[1:])] if lens is None else lens
    want, want_lse, o_tol, lse_tol = expected(q, k, v, starts, n, causal, scale or None)
    covered = ~want_lse.isnan()
    assert (o[~covered] == 7).all() and (lse[~covered] == 7).all()
    error, lse_error = (o.double() - want)[covered].abs(), (lse.double() - want_lse)[covered].abs()
    assert (error <= o_tol[covered]).all(), (error / o_tol[covered]).max()
    assert (lse_error <= lse_tol[covered]).all(), (lse_error / lse_tol[covered]).max()
    return o, lse


def ends(lens, first=0):
    out = [first]
    for n in lens:
        out.append(out[-1] + n)
    return out


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens, heads, kv_heads, dim, dtype", [
    ([1], 1, 1, 64, BF), ([1], 8, 2, 128, HF), ([77], 8, 2, 64, BF), ([128], 2, 2, 128, BF), ([129], 2, 2, 128, BF), ([256], 1, 1, 128, BF), ([257], 1, 1, 64, HF),
    ([127, 128, 129, 255, 256, 257], 2, 1, 128, BF), ([1, 1, 1, 1, 1], 4, 4, 128, HF), ([0, 5, 0, 0, 300, 0], 6, 2, 64, BF), ([640], 4, 4, 128, BF),
    ([100, 3, 900], 7, 1, 128, BF), ([33, 500], 40, 5, 64, HF), ([700, 20], 28, 4, 64, HF), ([250], 16, 1, 128, BF), ([40, 41], 100, 1, 128, BF), ([70], 128, 1, 64, BF),
    ([1300], 3, 1, 128, HF), ([5] * 60, 8, 2, 128, BF), ([2000, 1, 1999], 4, 2, 64, BF), ([17] * 9, 10, 10, 64, HF)])
def test_lengths_heads_types(lens, heads, kv_heads, dim, dtype, causal):
    check(*tensors(sum(lens), heads, kv_heads, dim, dtype, seed=sum(lens)), ends(lens), causal=causal)


@pytest.mark.parametrize("dim", [64, 128])
def test_a_long_prompt(dim):
    check(*tensors(9000, 4, 2, dim, BF, seed=dim), [0, 9000])


def test_many_sequences():
    r = torch.Generator().manual_seed(1)
    lens = torch.randint(0, 12, (3000,), generator=r).tolist()
    q, k, v = tensors(sum(lens), 2, 1, 64, BF, seed=2)
    o, lse, status = run(q, k, v, ends(lens))
    # (all sequences at once: tokens of one are those with its number)
    number = torch.repeat_interleave(torch.arange(3000), torch.tensor(lens)).cuda()
    for first in range(0, sum(lens), 1000):
        at = slice(first, min(first + 1000, sum(lens)))
        lo, hi = max(0, first - 12), at.stop
        sees = (number[at, None] == number[None, lo:hi]) & (torch.arange(lo, hi, device="cuda") <= torch.arange(at.start, at.stop, device="cuda")[:, None])
        for h in range(2):
            x = (q[h, at].double() @ k[0, lo:hi].double().t() / 8.0).masked_fill(~sees, -math.inf)
            w = torch.softmax(x, -1)
            tol = (w @ v[0, lo:hi].double().abs()) * (UNIT[BF] + 2.0 ** -15) + 2.0 ** -10 + (w @ v[0, lo:hi].double()).abs() * UNIT[BF]
            assert ((o[h, at].double() - w @ v[0, lo:hi].double()).abs() <= tol).all()
    assert status == [0, 0, 0, 0]


@pytest.mark.parametrize("order", ["hnd", "nhd"])
def test_tokens_of_no_sequence_and_strides(order):
    q, k, v = tensors(500, 6, 3, 64, BF, order, seed=3)
    check(q, k, v, [13, 200, 333])
    # heads and tokens with gaps, channels of a wider row
    wide = torch.randn((500, 12 * 3, 64), device="cuda").to(BF)
    q, k, v = (wide[:, i * 12:i * 12 + 12:s].transpose(0, 1) for i, s in ((0, 2), (1, 4), (2, 4)))
    check(q, k, v, [1, 100, 499], causal=False)


def test_padded_batch_with_nan_in_the_padding():
    q, k, v = tensors(4 * 150, 4, 2, 128, BF, seed=4)
    lens = [150, 1, 0, 77]
    for x in (q, k, v):
        for b, n in enumerate(lens):
            x[:, b * 150 + n:(b + 1) * 150] = math.nan
    for causal in (True, False):
        check(q, k, v, [0, 150, 300, 450, 600], lens, causal=causal)


@pytest.mark.parametrize("dtype", [BF, HF])
def test_scores_that_grow(dtype):
    q, k, v = tensors(1500, 4, 2, 64, dtype, seed=5, q_scale=4.0, ramp=6.0)
    check(q, k, v, [0, 1500])
    check(q, k, v, [0, 700, 1500], causal=False, scale=0.3)


@pytest.mark.parametrize("dtype, dim", [(BF, 128), (HF, 64)])
def test_every_row_tile_is_computed_again(dtype, dim):
    """Scores that rise by hundreds of bits along the sequence: several row tiles of every thread block overflow."""
    q, k, v = tensors(3500, 32, 4, dim, dtype, seed=13, q_scale=0.1)
    q[..., 0], k[..., 0] = 8.0, (torch.arange(3500, device="cuda") / 5.0).to(dtype)
    check(q, k, v, [0, 1700, 3500], scale=0.125)
    check(q, k, v, [0, 1700, 3500], causal=False, scale=0.125)


@pytest.mark.parametrize("dim, dtype", [(64, HF), (128, BF)])
def test_many_short_sequences_computed_again(dim, dtype):
    """Hundreds of row tiles a thread block, each of which goes into its chain once, however far apart the warps are that find it."""
    n, length = 4000, 48
    q, k, v = tensors(n * length, 2, 1, dim, dtype, seed=15)
    q[..., 0], k[..., 0] = 8.0, 0.0
    k.view(1, n, length, dim)[:, :, -4:, 0] = 400.0                     # the last keys: 2^577 times the first ones'
    v.view(1, n, length, dim)[:, ::3, 10, 5] = math.nan                 # and some of the values are seen by most rows only
    o, lse, status = run(q, k, v, list(range(0, (n + 1) * length, length)), scale=0.125)
    assert status == [0, 0, 0, 0]
    for b in (0, 1, 2, 1999, 2000, 3999):
        at = slice(b * length, (b + 1) * length)
        want, want_lse, tol, lse_tol = expected(q[:, at], k[:, at], v[:, at], [0], [length], True, 0.125)
        # (a value that is not finite in a place that a row does not see is NaN in the definition's product; the rows in front of it have none)
        clean = v[:, at].clone()
        clean[clean.isnan()] = 0.0
        want = expected(q[:, at], k[:, at], clean, [0], [length], True, 0.125)[0]
        tol = expected(q[:, at], k[:, at], clean, [0], [length], True, 0.125)[2]
        sees = torch.zeros_like(want, dtype=torch.bool)
        sees[:, 10:, 5] = b % 3 == 0
        assert torch.equal(o[:, at].isnan(), sees)
        assert ((o[:, at].double() - want).abs() <= tol)[~sees].all() and ((lse[:, at].double() - want_lse).abs() <= lse_tol).all()


@pytest.mark.parametrize("n", [17, 64, 100, 128])
def test_first_keys_at_minus_infinity_in_one_tile(n):
    """The reference is taken from the first 16 scores: a row in which all these are -infinity still has the others."""
    q, k, v = tensors(n, 2, 1, 64, BF, seed=16)
    q[..., 0], k[..., 0] = 1.0, -40.0
    k[:, :16, 0] = -math.inf
    o, lse, status = run(q, k, v, [0, n], scale=1.0)
    # (the tokens from 16 on are a sequence of their own)
    want, want_lse, tol, lse_tol = expected(q[:, 16:], k[:, 16:], v[:, 16:], [0], [n - 16], True, 1.0)
    assert status == [0, 0, 0, 0] and (o[:, :16] == 0).all() and (lse[:, :16] == -math.inf).all()
    assert ((o[:, 16:].double() - want).abs() <= tol).all() and ((lse[:, 16:].double() - want_lse).abs() <= lse_tol).all()


def test_long_sequences_of_small_row_tiles():
    """1,100 and 1,500 tokens with 128 heads on one key head: more row tiles than the planning kernel sorts by."""
    q, k, v = tensors(2605, 128, 1, 64, BF, seed=17)
    o, lse, status = run(q, k, v, ends([5, 1100, 1500]))
    assert status == [0, 0, 0, 0]
    some = [0, 63, 127]
    want, want_lse, tol, lse_tol = expected(q[some], k, v, ends([5, 1100, 1500])[:-1], [5, 1100, 1500], True)
    assert ((o[some].double() - want).abs() <= tol).all() and ((lse[some].double() - want_lse).abs() <= lse_tol).all()


def test_broadcast_heads_and_dimensions_of_one():
    q, k, v = tensors(300, 4, 1, 64, BF, seed=14)
    check(q, k.expand(4, -1, -1), v.expand(4, -1, -1), [0, 120, 300])    # one key head, repeated without a copy
    one = torch.randn(64 * 3, device="cuda").to(BF)
    q, k, v = (torch.as_strided(one, (1, 1, 64), (3, 5, 1), 64 * i) for i in range(3))
    out = torch.empty(64, dtype=BF, device="cuda").as_strided((1, 1, 64), (7, 9, 1))
    o = wb.prompt_attn(q, k, v, torch.tensor([0, 1], dtype=torch.int32, device="cuda"), o=out)
    assert torch.equal(o, v)                                            # one token: its own value


@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dim, heads, kv_heads", [(128, 2, 2), (64, 2, 2), (128, 16, 2)])
def test_values_that_a_token_does_not_see(what, dim, heads, kv_heads):
    """Tokens in front of a bad value or key have the results they have without it, within the definition's tolerance: the row tiles that meet
    it are computed again, with another reference and their sums in another order."""
    n = 700
    q, k, v = tensors(2 * n, heads, kv_heads, dim, BF, seed=6)
    clean, clean_lse = check(q, k, v, [0, n, 2 * n])
    want, want_lse, tol, lse_tol = expected(q, k, v, [0, n], [n, n], True)
    for at in (0, 5, 100, 127, 128, 300, n - 1):
        for t in (k, v):
            bad = t.clone()
            bad[:, at] = what
            if t is k and not math.isnan(what):
                bad[:, at, 1:] = t[:, at, 1:]                          # one channel: the score is + or - infinity
            o, lse, status = run(q, bad if t is k else k, bad if t is v else v, [0, n, 2 * n])
            assert status == [0, 0, 0, 0]
            assert ((lse.double() - want_lse).abs() <= lse_tol)[:, :at].all() and ((o.double() - want).abs() <= tol)[:, :at].all()
            assert torch.equal(o[:, n:], clean[:, n:]) and torch.equal(lse[:, n:], clean_lse[:, n:])      # the other sequence
            if t is v:
                assert ((lse.double() - want_lse).abs() <= lse_tol).all()
                assert (o[:, at:n].isnan() if math.isnan(what) else o[:, at:n] == what).all()
            elif math.isnan(what):
                assert o[:, at:n].isnan().all() and lse[:, at:n].isnan().all()
            else:
                seen = q[:, at:n, 0].float() * what                     # +infinity: NaN; -infinity: no such key
                assert (o[:, at:n].isnan().all(-1) == (seen == math.inf)).all() if at else True


def test_one_bad_channel_of_a_value():
    """The other channels of a row that sees it are what they were, up to the rounding of another way of adding."""
    q, k, v = tensors(300, 2, 1, 128, BF, seed=7)
    want, _, tol, _ = expected(q, k, v, [0], [300], True)
    v[:, 250, 3] = math.inf
    o, lse, status = run(q, k, v, [0, 300])
    assert (o[:, 250:, 3] == math.inf).all() and status == [0, 0, 0, 0]
    o[:, 250:, 3] = want[:, 250:, 3].to(BF)
    assert ((o.double() - want).abs() <= tol).all()


def test_rows_without_a_finite_score():
    q, k, v = tensors(200, 2, 1, 64, BF, seed=8)
    q[:, :, 0], k[:, :150, 0] = 1.0, -math.inf                          # scores of the first 150 keys: -infinity
    o, lse, status = run(q, k, v, [0, 200])
    assert (o[:, :150] == 0).all() and (lse[:, :150] == -math.inf).all() and status == [0, 0, 0, 0]
    assert o[:, 150:].isfinite().all() and lse[:, 150:].isfinite().all()
    want = v[0, 150].float()
    assert torch.equal(o[:, 150].float(), want.expand(2, -1))


def test_same_bits_again():
    q, k, v = tensors(3000, 8, 2, 128, BF, seed=9)
    starts = ends([700, 1, 1500, 299, 500])
    first = run(q, k, v, starts)
    for _ in range(4):
        again = run(q, k, v, starts)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_malformed_sequences():
    q, k, v = tensors(300, 2, 1, 64, BF, seed=10)
    for starts, lens, want in (([-5, 100, 300], None, [4, 100, 0, -5]), ([0, 100, 301], None, [4, 100, 1, 301]), ([0, 200, 100, 300], None, [4, 100, 1, 100]),
                               ([0, 100, 300], [100, 201], [4, 101, 1, 201]), ([0, 100, 300], [-1, 200], [4, 101, 0, -1])):
        o, lse, status = run(q, k, v, starts, lens)
        assert status == want
        alone = [(a, b - a) for i, (a, b) in enumerate(zip(starts, starts[1:])) if i != want[2]]
        if starts == [0, 200, 100, 300]:                                # (the third one begins in front of the second one's start)
            alone = alone[:1]
        want_o, _, tol, _ = expected(q, k, v, [a for a, _ in alone], [n for _, n in alone], True)
        covered = ~want_o.isnan()
        assert (o[~covered] == 7).all()
        assert ((o.double() - want_o).abs()[covered] <= tol[covered]).all()
    # many sequences that claim the same tokens, and starts far outside
    o, lse, status = run(q, k, v, [0, 300] * 1500 + [7, 50])
    assert status[:2] == [4, 100] and torch.equal(o, run(q, k, v, [0, 300])[0])
    o, lse, status = run(q, k, v, [0, 100, 10 ** 9, 100, 300, 299, 300])
    want_o, _, tol, _ = expected(q, k, v, [0, 100], [100, 200], True)
    assert status[:2] == [4, 100] and ((o.double() - want_o).abs() <= tol).all()


@pytest.mark.parametrize("bits", [13, 16, 20, 23, 24, 25])
def test_small_probabilities_of_fp16(bits):
    """One key in front with a value near zero, a thousand behind it with probabilities of 2^-bits of it: what they add is more than that value."""
    n = 1000
    q, k, v = tensors(n, 2, 1, 64, HF, seed=19, q_scale=0.02)
    q[..., 0], k[..., 0], k[:, 0, 0] = 1.0, 0.0, 8.0 * bits * math.log(2.0)
    v[:, 0] = v[:, 0] * 2.0 ** -10
    check(q, k, v, [0, n])
    check(q, k, v, [0, 100, n], causal=False)


@pytest.mark.parametrize("lens", [[300], [1] * 32, [0, 40, 0, 0, 200, 7, 0, 129], [100] * 9])
def test_one_launch_or_two_are_the_same(lens):
    """Few row tiles of 32 sequences at most are planned where they are computed; 33 sequences are not."""
    q, k, v = tensors(sum(lens), 8, 2, 64, BF, seed=18)
    few = run(q, k, v, ends(lens))
    assert wb.last_launch_count() == 1 and few[2] == [0, 0, 0, 0]
    many = run(q, k, v, ends(lens + [0] * (33 - len(lens))))
    assert wb.last_launch_count() == 2 and many[2] == [0, 0, 0, 0]
    assert torch.equal(few[0], many[0]) and torch.equal(few[1], many[1])


def test_captured_call_follows_the_lengths():
    q, k, v = tensors(1000, 8, 2, 128, BF, seed=11)
    start, length = torch.zeros(5, dtype=torch.int32, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    o, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        wb.prompt_attn(q, k, v, start, seq_len=length, o=o, lse=lse)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            wb.prompt_attn(q, k, v, start, seq_len=length, o=o, lse=lse)
    torch.cuda.synchronize()
    for starts, lens in (([0, 250, 500, 750, 1000], [250, 1, 0, 249]), ([0, 0, 0, 1000, 1000], [0, 0, 1000, 0])):
        start.copy_(torch.tensor(starts)), length.copy_(torch.tensor(lens))
        graph.replay()
        want, want_lse, _ = run(q, k, v, starts, lens)
        for b, n in enumerate(lens):
            at = slice(starts[b], starts[b] + n)
            assert torch.equal(o[:, at], want[:, at]) and torch.equal(lse[:, at], want_lse[:, at])


def test_two_calls_at_once():
    jobs = [(tensors(2500, 4, 2, d, BF, seed=d), ends([1200, 1300])) for d in (64, 128)]
    want = [run(*t, s) for t, s in jobs]
    streams = [torch.cuda.Stream() for _ in jobs]
    starts = [torch.tensor(s, dtype=torch.int32, device="cuda") for _, s in jobs]
    torch.cuda.synchronize()
    got = [[wb.prompt_attn(*t, start, return_lse=True, stream=stream) for (t, _), start, stream in zip(jobs, starts, streams)] for _ in range(5)]
    torch.cuda.synchronize()
    for turn in got:
        for (o, lse), w in zip(turn, want):
            assert torch.equal(o, w[0]) and torch.equal(lse, w[1])


def test_offsets_behind_two_to_the_31():
    tokens, row = 140000, 16384                                         # 2.3e9 elements
    buf = torch.zeros((tokens, row), dtype=BF, device="cuda")
    x = buf[:, :4 * 128].view(tokens, 4, 128).transpose(0, 1)
    tail = torch.randn((4, 300, 128), device="cuda").to(BF)
    x[:, -300:] = tail
    starts = [0, 3, tokens - 300, tokens - 300, tokens]
    starts = [tokens - 310, tokens - 300, tokens]
    o, lse, status = run(x, x[:2], x[2:], starts)
    want, want_lse, tol, lse_tol = expected(tail, tail[:2], tail[2:], [0], [300], True)
    assert status == [0, 0, 0, 0]
    assert ((o[:, -300:].double() - want).abs() <= tol).all() and ((lse[:, -300:].double() - want_lse).abs() <= lse_tol).all()


def test_a_wait_that_runs_out():
    q, k, v = tensors(3000, 4, 2, 128, BF, seed=12)
    _, _, status = run(q, k, v, [0, 3000], flags=wb.PROMPT_SELFTEST_LOST_TILE)
    assert status[0] == wb.ERR_TIMEOUT and 110 <= status[1] <= 131 and status[2] == 0
    check(q, k, v, [0, 3000])
