"""Attention of whole prompts where test_gpu_prompt_attn.py looks at NaN and infinities alone: every finite result beside them against the definition in 64
bits, with the tolerances derived there; results in a buffer of their own layout."""
import math

import pytest
import torch

from paper_2609_34814_b200 import binding as wb
from test_gpu_prompt_attn import BF, HF, ends, expected, run, tensors

pytestmark = pytest.mark.gpu


def without(q, k, v, dead, causal, scale):
    """The definition (o, lse, tolerances) for one sequence [heads, n, dim] where the keys of dead [heads, n rows, n keys] have scores of -infinity; k is
    finite.  Rows that see no other key: o = 0, lse = -infinity."""
    heads, n, dim = q.shape
    group = heads // k.shape[0]
    unit = torch.finfo(q.dtype).eps / 2
    o, lse, o_tol, lse_tol = [], [], [], []
    for h in range(heads):
        qh, kh, vh = q[h].double(), k[h // group].double(), v[h // group].double()
        hidden = dead[h].clone()
        if causal:
            hidden |= torch.ones((n, n), dtype=torch.bool, device="cuda").triu(1)
        x = (qh @ kh.t() * scale).masked_fill(hidden, -math.inf)
        size = (qh.abs() @ kh.abs().t() * scale).masked_fill(hidden, 0.0)
        none = hidden.all(-1)
        w = torch.softmax(x.masked_fill(none[:, None], 0.0), -1).masked_fill(none[:, None], 0.0)
        e = (dim + 2) * 2.0 ** -24 * size.amax(-1) + 2.0 ** -20
        o.append(w @ vh), lse.append(torch.logsumexp(x, -1))
        lse_tol.append((e + 2.0 ** -22 * lse[-1].abs()).masked_fill(none, 0.0))
        tol = (w @ vh.abs()) * (unit + 2 * e)[:, None] + o[-1].abs() * unit + 2.0 ** -24
        if q.dtype == HF:
            tol = tol + 2.0 ** -25 * (~hidden).double() @ vh.abs()
        o_tol.append(tol.masked_fill(none[:, None], 0.0))
    return tuple(torch.stack(t) for t in (o, lse, o_tol, lse_tol))


def compare(o, lse, want, want_lse, tol, lse_tol, rows=None):
    rows = torch.ones(lse.shape, dtype=torch.bool, device="cuda") if rows is None else rows
    none = want_lse == -math.inf
    assert (lse[none & rows] == -math.inf).all() and (o[none & rows] == 0).all()
    rows = rows & ~none
    assert ((o.double() - want).abs() <= tol)[rows].all(), ((o.double() - want).abs() / tol)[rows].max()
    assert ((lse.double() - want_lse).abs() <= lse_tol)[rows].all()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dim, heads, kv_heads, dtype", [(128, 2, 2, BF), (64, 2, 2, HF), (128, 16, 2, HF), (64, 6, 1, BF)])
@pytest.mark.parametrize("sign", [1, -1])
def test_a_key_with_an_infinite_channel(dim, heads, kv_heads, dtype, causal, sign):
    """Rows whose score for that key is -infinity have the results of the other keys; where it is +infinity they are NaN.  (A query's first channel is never
    zero here.)"""
    n = 700
    q, k, v = tensors(2 * n, heads, kv_heads, dim, dtype, seed=21)
    q[..., 0] += (q[..., 0] == 0).to(dtype)
    clean, clean_lse, _ = run(q, k, v, [0, n, 2 * n], causal=causal)
    for at in (0, 5, 100, 127, 128, 300, 640, n - 1):
        bad = k.clone()
        bad[:, at, 0] = sign * math.inf
        o, lse, status = run(q, bad, v, [0, n, 2 * n], causal=causal)
        assert status == [0, 0, 0, 0] and torch.equal(o[:, n:], clean[:, n:]) and torch.equal(lse[:, n:], clean_lse[:, n:])
        down = sign * q[:, :n, 0].float() < 0
        dead = torch.zeros((heads, n, n), dtype=torch.bool, device="cuda")
        dead[:, :, at] = down
        sees = torch.ones((heads, n), dtype=torch.bool, device="cuda")
        if causal:
            sees[:, :at] = False
        up = sees & ~down
        assert o[:, :n][up].isnan().all() and lse[:, :n][up].isnan().all()
        compare(o[:, :n], lse[:, :n], *without(q[:, :n], k[:, :n], v[:, :n], dead, causal, 1.0 / math.sqrt(dim)), rows=~up)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n, first, dim, dtype", [(200, 150, 64, BF), (200, 128, 128, HF), (700, 129, 128, BF), (700, 256, 64, HF), (700, 300, 128, BF), (900, 512, 64, BF),
                                                  (900, 899, 128, HF), (300, 300, 64, BF)])
def test_first_keys_at_minus_infinity(n, first, dim, dtype, causal):
    """The first keys' scores are all -infinity, whole key tiles of them: the second computation's reference comes from a later tile."""
    q, k, v = tensors(n, 6, 2, dim, dtype, seed=22)
    q[..., 0], k[..., 0] = 1.0, 0.0
    bad = k.clone()
    bad[:, :first, 0] = -math.inf
    o, lse, status = run(q, bad, v, [0, n], causal=causal)
    assert status == [0, 0, 0, 0]
    dead = torch.zeros((6, n, n), dtype=torch.bool, device="cuda")
    dead[:, :, :first] = True
    compare(o, lse, *without(q, k, v, dead, causal, 1.0 / math.sqrt(dim)))


@pytest.mark.parametrize("dim, dtype", [(64, HF), (128, BF)])
def test_keys_at_minus_infinity_in_the_middle(dim, dtype):
    """Whole tiles of them behind the first, then scores that outgrow the first ones."""
    n = 900
    q, k, v = tensors(n, 4, 2, dim, dtype, seed=23, q_scale=0.5)
    q[..., 0], k[..., 0] = 8.0, 0.0
    k[:, 600:, 0] = 60.0
    bad = k.clone()
    bad[:, 100:520, 0] = -math.inf
    o, lse, status = run(q, bad, v, [0, n])
    assert status == [0, 0, 0, 0]
    dead = torch.zeros((4, n, n), dtype=torch.bool, device="cuda")
    dead[:, :, 100:520] = True
    compare(o, lse, *without(q, k, v, dead, True, 1.0 / math.sqrt(dim)))


@pytest.mark.parametrize("repeat", [False, True])
def test_results_behind_two_to_the_31(repeat):
    """o by itself lies in rows of 16,384 elements, so that its last tokens' elements are more than 2^31 behind its first, in the first computation and in
    the second (which scores that outgrow the first ones cause)."""
    tokens, row, heads, n = 140000, 16384, 4, 300
    q, k, v = tensors(tokens, heads, 2, 128, BF, seed=24)
    if repeat:
        q[..., 0], k[..., 0] = 8.0, 0.0
        k[:, -50:, 0] = 200.0
    buf = torch.full((tokens, row), 7.0, dtype=BF, device="cuda")
    o = buf[:, :heads * 128].view(tokens, heads, 128).transpose(0, 1)
    assert (tokens - n) * o.stride(1) > 2 ** 31
    lse, status = torch.full((heads, tokens), 7.0, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    starts = [tokens - n - 10, tokens - n, tokens]
    wb.prompt_attn(q, k, v, torch.tensor(starts, dtype=torch.int32, device="cuda"), o=o, lse=lse, dev_status=status)
    assert status.tolist() == [0, 0, 0, 0]
    for a, b in zip(starts, starts[1:]):
        want, want_lse, tol, lse_tol = expected(q[:, a:b], k[:, a:b], v[:, a:b], [0], [b - a], True)
        compare(o[:, a:b], lse[:, a:b], want, want_lse, tol, lse_tol)
    assert (lse[:, :starts[0]] == 7).all() and (buf[:, heads * 128:] == 7).all() and (buf[:starts[0]] == 7).all()


@pytest.mark.parametrize("order", ["nhd", "hnd"])
def test_one_buffer_for_inputs_and_results(order):
    """q, k, v and o side by side in the rows of one buffer; o one row too early is refused."""
    heads, kv_heads, dim, lens = 6, 2, 64, [200, 77]
    q, k, v = tensors(sum(lens), heads, kv_heads, dim, BF, seed=25)
    want = run(q, k, v, ends(lens))
    parts = [heads, kv_heads, kv_heads, heads]
    if order == "nhd":
        buf = torch.full((sum(lens), sum(parts), dim), 7.0, dtype=BF, device="cuda").transpose(0, 1)
    else:
        buf = torch.full((sum(parts), sum(lens), dim), 7.0, dtype=BF, device="cuda")
    x, y, z, o = buf.split(parts)
    x.copy_(q), y.copy_(k), z.copy_(v)
    start = torch.tensor(ends(lens), dtype=torch.int32, device="cuda")
    _, lse = wb.prompt_attn(x, y, z, start, o=o, return_lse=True)
    assert torch.equal(o, want[0]) and torch.equal(lse, want[1]) and torch.equal(x, q) and torch.equal(y, k) and torch.equal(z, v)
    before = buf.clone()
    for early in (1, kv_heads, kv_heads + 1, 2 * kv_heads + 1):
        with pytest.raises(wb.WavealError) as e:
            wb.prompt_attn(x, y, z, start, o=buf[sum(parts[:3]) - early:sum(parts) - early])
        assert e.value.status == wb.ERR_INVALID_ARG
    assert torch.equal(buf, before)


@pytest.mark.parametrize("dim, dtype, bits", [(64, HF, 10), (64, HF, 40), (128, BF, 40), (128, BF, 300)])
def test_an_infinite_value_with_a_small_probability(dim, dtype, bits):
    """2^-bits of the largest one: the rows that see it have an infinity there, or NaN where the probability rounds to zero; nothing else changes."""
    n = 400
    q, k, v = tensors(n, 4, 2, dim, dtype, seed=26, q_scale=0.02)
    q[..., 0], k[..., 0], k[:, 0, 0] = 8.0, 0.0, bits * math.log(2.0) * math.sqrt(dim) / 8.0
    want, want_lse, tol, lse_tol = expected(q, k, v, [0], [n], True)
    v[:, 150, 3] = math.inf
    o, lse, status = run(q, k, v, [0, n])
    assert status == [0, 0, 0, 0]
    seen = o[:, 150:, 3]
    assert ((seen == math.inf) | seen.isnan()).all() and ((seen == math.inf).all() if bits == 10 else True)
    o[:, 150:, 3] = want[:, 150:, 3].to(dtype)
    compare(o, lse, want, want_lse, tol, lse_tol)


def test_results_between_the_heads_of_one_buffer():
    """Every other head of the buffer's rows is q's or o's, every fourth k's or v's: one stride in common, no element."""
    lens = [200, 1, 99]
    q, k, v = tensors(sum(lens), 6, 3, 64, BF, seed=27)
    want = run(q, k, v, ends(lens))
    wide = torch.full((sum(lens), 36, 64), 7.0, dtype=BF, device="cuda")
    x, y, z, o = (wide[:, a:b:s].transpose(0, 1) for a, b, s in ((0, 12, 2), (12, 24, 4), (24, 36, 4), (1, 12, 2)))
    x.copy_(q), y.copy_(k), z.copy_(v)
    start = torch.tensor(ends(lens), dtype=torch.int32, device="cuda")
    wb.prompt_attn(x, y, z, start, o=o)
    assert torch.equal(o, want[0]) and torch.equal(x, q) and torch.equal(y, k) and torch.equal(z, v) and (wide[:, 13:24:4] == 7).all()
    # one key head, repeated without a copy, in front of o in every row
    y, z = (t[:1].expand(6, -1, -1) for t in (y, z))
    want = run(q, k[:1], v[:1], ends(lens))
    wb.prompt_attn(x, y, z, start, o=wide[:, 25:36:2].transpose(0, 1)[:6])
    assert torch.equal(wide[:, 25:36:2].transpose(0, 1), want[0])
    with pytest.raises(wb.WavealError):
        wb.prompt_attn(x, y, z, start, o=wide[:, 24:36:2].transpose(0, 1))
