"""A clip and its continuations through rotation, block-sparse attention, cache and prefix attention, against the
definitions in 64 bits."""
import math

import pytest
import torch

from paper_2609_34814_b200 import continue_clip as cc
from tests.serving_util import rotated


@pytest.mark.gpu
def test_clip_and_continuations():
    heads, dim, grid, frames, new_frames, ways = 2, 64, (5, 9), 5, 2, 3
    layer = cc.ClipLayer(heads, dim, grid, frames, new_frames, ways, page=16)
    g = torch.Generator().manual_seed(3)
    draw = lambda n: [torch.randn((heads, n, dim), generator=g).bfloat16() for _ in range(3)]  # noqa: E731
    theta = layer.freqs.cpu().double() / 2.0 ** 64 * (2 * math.pi)
    # (what the library rotates is rounded to bf16, as the keys in the cache are)
    turn = lambda x, pos: rotated(x.double(), pos.cpu(), theta, layer.axis_pairs, True).bfloat16().double()  # noqa: E731
    q, k, v = draw(layer.clip)
    blocks = -(-layer.clip // 64)
    mask = cc.band_mask(heads, blocks, 1)
    o = layer.start(q.cuda(), k.cuda(), v.cuda(), mask).double().cpu()
    pos = layer.positions(0, frames)
    qr, kr = turn(q, pos), turn(k, pos)
    bits = (mask[0].cpu()[:, :, None] >> torch.arange(64) & 1).bool().view(blocks, -1)[:, :blocks]
    seen = bits.repeat_interleave(64, 0).repeat_interleave(64, 1)[:layer.clip, :layer.clip]
    x = (qr @ kr.transpose(1, 2) / math.sqrt(dim)).masked_fill(~seen, -math.inf)
    # p in bf16 (2^-8 of the mean of |v|), the result in bf16; a rotated channel that falls on the other side of a bf16 step moves
    # a score by 2^-8 |q k| of one channel, some of which add up at random: 2^-8 more
    def close(got, w, values):
        want = w @ values
        bound = (w @ values.abs()) * 2.0 ** -6 + want.abs() * 2.0 ** -8 + 1e-6
        assert bool(((got - want).abs() <= bound).all()), float(((got - want).abs() - bound).max())
    close(o, torch.softmax(x, -1), v.double())
    own_k, own_v = [[] for _ in range(ways)], [[] for _ in range(ways)]
    for f in range(new_frames):
        q, k, v = draw(ways * layer.frame)
        o = layer.step(q.cuda(), k.cuda(), v.cuda()).double().cpu()
        pos = layer.positions(frames + f, 1)
        for w in range(ways):
            part = slice(w * layer.frame, (w + 1) * layer.frame)
            own_k[w].append(turn(k[:, part], pos))
            own_v[w].append(v[:, part].double())
            keys, values = torch.cat([kr] + own_k[w], 1), torch.cat([clip_v(layer)] + own_v[w], 1)
            close(o[:, part], torch.softmax(turn(q[:, part], pos) @ keys.transpose(1, 2) / math.sqrt(dim), -1), values)
    assert layer.status.tolist() == [0] * 4


def clip_v(layer):
    """the clip's values, as the cache holds them"""
    n = layer.clip
    return layer.cache.v[layer.clip_pages.long()].transpose(0, 1).reshape(layer.heads, -1, layer.head_dim)[:, :n].double().cpu()


@pytest.mark.gpu
def test_command_runs(capsys):
    cc.main(["--heads", "2", "--frames", "2", "--height", "6", "--width", "10", "--continuations", "3"])
    out = capsys.readouterr().out
    assert "frame 1: 3 continuations over 240 keys" in out


@pytest.mark.gpu
def test_a_refused_frame_leaves_the_layer_as_it_was():
    heads, dim, grid, ways = 1, 64, (5, 9), 2
    layer = cc.ClipLayer(heads, dim, grid, 2, 2, ways, page=16)
    draw = lambda n: [torch.randn((heads, n, dim), device="cuda").bfloat16() for _ in range(3)]  # noqa: E731
    layer.start(*draw(layer.clip), cc.band_mask(heads, 2, 1))
    layer.step(*draw(ways * layer.frame))
    with pytest.raises(ValueError):                               # refused by the append: queries of another head_dim
        q, k, v = draw(ways * layer.frame)
        layer.step(q[..., :32], k, v)
    assert layer.seen == 1
    layer.step(*draw(ways * layer.frame))
    kept = layer.cache.k.clone()
    for _ in range(2):
        with pytest.raises(ValueError):                           # no pages left
            layer.step(*draw(ways * layer.frame))
        assert layer.seen == 2
    assert torch.equal(layer.cache.k.isnan(), kept.isnan()) and torch.equal(layer.cache.k.nan_to_num(), kept.nan_to_num())
    assert layer.status.tolist() == [0] * 4
