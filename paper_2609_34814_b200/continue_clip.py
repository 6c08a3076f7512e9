"""One attention layer of a model that continues a clip in several ways: the calls of this library as they follow each other.

  python -m paper_2609_34814_b200.continue_clip [--heads 8] [--frames 6] [--new-frames 2] [--continuations 4]

The clip so far goes through the block-sparse attention in its planned order, on queries and keys rotated by frame, height and
width, and its keys and values into the paged cache, once.  Every continuation then adds frame after frame: the frame's keys are rotated
on their way into the continuation's own pages, the queries beside them, and all continuations attend to the shared clip and to their
own frames in one call.  A model would put its projections and its other layers around this; here the queries, keys and values are drawn.
"""
from __future__ import annotations

import argparse

import torch

from . import binding as wb


class ClipLayer:
    """Cache, rotation and page tables of one layer.  heads: query and key heads; grid: a frame's tokens (height, width);
    clip_frames: frames of the shared clip; new_frames: room for every continuation's own."""

    def __init__(self, heads, head_dim, grid, clip_frames, new_frames, continuations, page=64, device="cuda"):
        self.heads, self.head_dim, self.grid, self.page = heads, head_dim, grid, page
        self.frame = grid[0] * grid[1]
        self.clip = clip_frames * self.frame
        self.continuations, self.new_frames, self.device = continuations, new_frames, device
        shared, own = -(-self.clip // page), -(-new_frames * self.frame // page)
        shape = (shared + own * continuations, heads, page, head_dim)
        self.cache = wb.PagedCache(*(torch.empty(shape, dtype=torch.bfloat16, device=device) for _ in range(2)))
        pages = torch.arange(shape[0], dtype=torch.int32, device=device)
        self.clip_pages, self.table = pages[:shared], pages[shared:].view(continuations, own)
        pairs = head_dim // 2
        self.axis_pairs = [pairs - 2 * (pairs // 3), pairs // 3, pairs // 3]
        self.freqs = torch.cat([wb.rope_freqs(2 * n, device=device)[0] for n in self.axis_pairs])
        self.seen = 0                                    # own frames of every continuation
        self.status = torch.zeros(4, dtype=torch.int32, device=device)

    def positions(self, first_frame, frames):
        """frame, height and width of `frames` whole frames' tokens"""
        t = torch.arange(frames * self.frame, device=self.device)
        f, rest = first_frame + t // self.frame, t % self.frame
        return torch.stack([f, rest // self.grid[1], rest % self.grid[1]]).to(torch.int32)

    def start(self, q, k, v, mask_bits, block=64):
        """Attention of the clip to itself under a block mask (bitmap [heads, blocks, words]); keeps its keys and values.
        q, k, v: [heads, tokens, head_dim]."""
        blocks = -(-self.clip // block)
        row_ptr, indices = wb.bitmap_to_csr(mask_bits, blocks)
        plan = wb.plan_bitmap(wb.plan_desc_default(heads=self.heads, n_q_blocks=blocks, n_kv_blocks=blocks), mask_bits)
        positions = self.positions(0, self.clip // self.frame)
        start = torch.tensor([0, self.clip], dtype=torch.int32, device=self.device)
        # the clip is a batch of one whose own pages are the ones that all continuations will share
        q = wb.cache_append(self.cache, k, v, start, start[1:], self.clip_pages[None], positions=positions, freqs=self.freqs, q=q,
                            interleaved=True, axis_pairs=self.axis_pairs, dev_status=self.status)
        k, _ = wb.rope(k, positions, self.freqs, interleaved=True, axis_pairs=self.axis_pairs)
        o = torch.empty_like(q)
        desc = wb.attn_desc(q, k, v, o, self.clip, self.clip, block)
        wb.bsattn_fwd(desc, q, k, v, o, row_ptr, indices, row_order=plan.row_order, dev_status=self.status)
        return o

    def step(self, q, k, v):
        """The next frame of every continuation: q, k, v [heads, continuations * frame tokens, head_dim], one continuation after
        another.  Returns their attention output, laid out the same."""
        B = self.continuations
        start = torch.arange(B + 1, dtype=torch.int32, device=self.device) * self.frame
        if self.seen >= self.new_frames:
            raise ValueError("no pages left for another frame")
        positions = self.positions(self.clip // self.frame + self.seen, 1).repeat(1, B)
        kept = torch.full((B,), (self.seen + 1) * self.frame, dtype=torch.int32, device=self.device)
        q = wb.cache_append(self.cache, k, v, start, kept, self.table, positions=positions, freqs=self.freqs, q=q, prefix_len=self.clip,
                            interleaved=True, axis_pairs=self.axis_pairs, dev_status=self.status)
        # (a frame's tokens see each other: no causal mask inside it)
        o = wb.prefix_attn(self.cache, q, start, kept, self.table, self.clip_pages, self.clip, causal=False, dev_status=self.status)
        self.seen += 1                                   # (a refused frame is not counted)
        return o


def band_mask(heads, blocks, width, device="cuda"):
    """bitmap of a band of blocks around the diagonal and the first block for all"""
    i = torch.arange(blocks)
    m = ((i[:, None] - i[None]).abs() <= width) | (i[None] == 0)
    words = -(-blocks // 64)
    bits = torch.zeros((blocks, words * 64), dtype=torch.bool)
    bits[:, :blocks] = m
    value = (bits.view(blocks, words, 64).long() << torch.arange(64)).sum(-1)
    return value[None].expand(heads, -1, -1).contiguous().to(device)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("heads", 8), ("head-dim", 128), ("height", 30), ("width", 52), ("frames", 6), ("new-frames", 2), ("continuations", 4)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args(argv)
    layer = ClipLayer(a.heads, a.head_dim, (a.height, a.width), a.frames, a.new_frames, a.continuations)
    g = torch.Generator(device="cuda").manual_seed(0)
    draw = lambda n: (torch.randn((a.heads, n, a.head_dim), generator=g, device="cuda").bfloat16() for _ in range(3))  # noqa: E731
    o = layer.start(*draw(layer.clip), band_mask(a.heads, -(-layer.clip // 64), 8))
    print(f"clip: {layer.clip} tokens, {a.heads} heads, mean |o| {o.float().abs().mean().item():.4f}")
    for f in range(a.new_frames):
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        q, k, v = draw(a.continuations * layer.frame)
        begin.record()
        o = layer.step(q, k, v)
        end.record()
        torch.cuda.synchronize()
        keys = layer.clip + layer.seen * layer.frame
        flops = 4 * a.heads * a.head_dim * q.shape[1] * keys
        print(f"frame {f}: {a.continuations} continuations over {keys} keys, {begin.elapsed_time(end) * 1e3:.0f} us "
              f"({flops / begin.elapsed_time(end) / 1e9:.0f} TFLOP/s, append included), mean |o| {o.float().abs().mean().item():.4f}")
    code = layer.status.tolist()
    if code[0]:
        raise SystemExit(f"device status {code}")


if __name__ == "__main__":
    main()
