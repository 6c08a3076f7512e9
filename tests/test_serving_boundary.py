"""Host-only checks of the rotary, cache and prefix-attention entry points: struct layouts, frequency tables, refusals
(all before any CUDA work, so they run without a GPU)."""
import ctypes
import math

import pytest
import torch

from paper_2609_34814_b200 import binding as wb
from paper_2609_34814_b200 import build as wbuild


@pytest.fixture(scope="module")
def lib():
    wbuild.build()
    return wb.load()


def test_struct_layouts():
    assert ctypes.sizeof(wb.Rotation) == 32
    assert ctypes.sizeof(wb.RopeDesc) == 120 and wb.RopeDesc.rot.offset == 20 and wb.RopeDesc.q_stride.offset == 56
    assert ctypes.sizeof(wb.CacheDesc) == 72 and wb.CacheDesc.k_stride.offset == 24
    assert ctypes.sizeof(wb.BatchDesc) == 32 and wb.BatchDesc.table_stride.offset == 24
    assert ctypes.sizeof(wb.AppendStrides) == 64
    # what the binding packs is laid out the same
    assert (wb._ROTATION.size, wb._ROPE.size, wb._CACHE.size, wb._BATCH.size, wb._STRIDES.size) == (32, 120, 72, 32, 64)
    d = wb.RopeDesc.from_buffer_copy(wb._ROPE.pack(1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12, 1.5, 21, 22, 23, 24, 25, 26, 27, 28))
    assert (d.tokens, d.dtype, d.rot.rot_dim, d.rot.axis_pairs[2], d.rot.inverse, d.rot.amplitude) == (1, 5, 6, 11, 12, 1.5)
    assert (d.q_stride[0], d.q_out_stride[1], d.k_out_stride[1]) == (21, 24, 28)
    c = wb.CacheDesc.from_buffer_copy(wb._CACHE.pack(1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11))
    assert (c.n_pages, c.page_size, c.kv_heads, c.head_dim, c.dtype, c.k_stride[0], c.v_stride[2]) == (1, 2, 3, 4, 5, 6, 11)
    b = wb.BatchDesc.from_buffer_copy(wb._BATCH.pack(1, 2, 3, 4, 5, 6, 7))
    assert (b.batch, b.tokens, b.q_heads, b.max_pages, b.prefix_len, b.flags, b.table_stride) == (1, 2, 3, 4, 5, 6, 7)


@pytest.mark.parametrize("rot", [2, 8, 64, 128])
def test_frequencies(lib, rot):
    def theta(*a, **k):
        f, amplitude = wb.rope_freqs(rot, *a, device="cpu", **k)
        return [int(x) * math.pi / 2 ** 63 for x in f.tolist()], amplitude
    plain = [10000.0 ** (-2 * i / rot) for i in range(rot // 2)]
    near = lambda a, b: all(abs(x - y) <= 1e-15 * y + 2.0 ** -60 for x, y in zip(a, b))  # noqa: E731
    assert near(theta()[0], plain) and theta()[1] == 1.0
    assert near(theta(scaling="linear", factor=8.0)[0], [x / 8 for x in plain])
    ntk, _ = theta(scaling="ntk", factor=8.0)
    if rot > 2:
        assert abs(ntk[0] - 1.0) < 1e-14 and abs(ntk[-1] - plain[-1] / 8) < 1e-14 * plain[-1]     # fastest kept, slowest stretched
    parts, amplitude = theta(500000.0, "parts", 16.0, 8192)
    assert abs(amplitude - (0.1 * math.log(16.0) + 1)) < 1e-6
    for i, t in enumerate(parts):
        raw = 500000.0 ** (-2 * i / rot)
        turns = 8192 * raw / (2 * math.pi)
        want = raw if turns >= 32 else raw / 16 if turns <= 1 else raw * (turns - 1) / 31 + raw / 16 * (32 - turns) / 31
        assert abs(t - want) <= 1e-14 * want + 2.0 ** -60


@pytest.mark.parametrize("args", [(0, 1e4, 0, 1.0, 0), (3, 1e4, 0, 1.0, 0), (8, 1.0, 0, 1.0, 0), (8, math.nan, 0, 1.0, 0), (8, math.inf, 0, 1.0, 0),
                                  (8, 1e4, 4, 1.0, 0), (8, 1e4, -1, 1.0, 0), (8, 1e4, 1, 0.5, 0), (8, 1e4, 2, math.nan, 0), (8, 1e4, 3, 2.0, 0)])
def test_frequencies_refused(lib, args):
    buf = (ctypes.c_int64 * 8)()
    rot, base, scaling, factor, trained = args
    assert lib.waveal_rope_freqs(rot, base, scaling, factor, trained, ctypes.addressof(buf), None) == wb.ERR_INVALID_ARG
    assert lib.waveal_rope_freqs(8, 1e4, 0, 1.0, 0, None, None) == wb.ERR_INVALID_ARG


def rope_desc(**kw):
    d = wb.RopeDesc()
    d.tokens, d.head_dim, d.q_heads, d.k_heads, d.dtype = 4, 64, 2, 1, wb.BF16
    d.rot = wb.Rotation(64, 0, 1, (32, 0, 0), 0, 1.0)
    d.q_stride = d.q_out_stride = d.k_stride = d.k_out_stride = (256, 64)
    for k, v in kw.items():
        setattr(d.rot if hasattr(d.rot, k) else d, k, v)
    return d


@pytest.mark.parametrize("kw, status", [
    (dict(tokens=-1), 1), (dict(q_heads=0), 1), (dict(k_heads=-1), 1), (dict(q_heads=1 << 21), 2), (dict(head_dim=1), 2),
    (dict(head_dim=513), 2), (dict(dtype=3), 2), (dict(dtype=-1), 2), (dict(rot_dim=63), 1), (dict(rot_dim=0), 1), (dict(rot_dim=66), 1),
    (dict(pairs=2), 1), (dict(axes=0), 1), (dict(axes=4), 1), (dict(axis_pairs=(31, 0, 0)), 1), (dict(axis_pairs=(31, 1, 0)), 1),
    (dict(axes=2, axis_pairs=(33, -1, 0)), 1), (dict(amplitude=math.nan), 1), (dict(amplitude=math.inf), 1)])
def test_rope_refused(lib, kw, status):
    d = rope_desc(**kw)
    assert lib.waveal_rope(ctypes.byref(d), 0x1000, 0x2000, 0x3000, 0x4000, 0x5000, 0x6000, None) == status
    assert wb.last_error()


def test_rope_refuses_pointers(lib):
    d = rope_desc()
    good = [0x1000, 0x2000, 0x3000, 0x4000, 0x5000, 0x6000]
    for i in range(6):
        assert lib.waveal_rope(ctypes.byref(d), *[None if i == j else p for j, p in enumerate(good)], None) == wb.ERR_INVALID_ARG
    assert lib.waveal_rope(None, *good, None) == wb.ERR_INVALID_ARG
    assert lib.waveal_rope(ctypes.byref(d), 0x1001, *good[1:], None) == wb.ERR_INVALID_ARG
    d.q_out_stride[1] = 128
    assert lib.waveal_rope(ctypes.byref(d), 0x1000, 0x1000, *good[2:], None) == wb.ERR_INVALID_ARG
    d = rope_desc(tokens=0)
    assert lib.waveal_rope(ctypes.byref(d), None, None, None, None, None, None, None) == wb.OK


def cache_desc(**kw):
    d = wb.CacheDesc(10, 16, 2, 128, wb.BF16, (4096, 2048, 128), (4096, 2048, 128))
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def batch_desc(**kw):
    d = wb.BatchDesc(3, 3, 4, 5, 100, 0, 5)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


BAD_CACHE = [(dict(n_pages=0), 1), (dict(kv_heads=0), 1), (dict(page_size=8), 2), (dict(page_size=48), 2), (dict(page_size=1 << 17), 2),
             (dict(kv_heads=1 << 21), 2), (dict(dtype=wb.FP32), 2)]
BAD_BATCH = [(dict(batch=-1), 1), (dict(tokens=-1), 1), (dict(max_pages=-1), 1), (dict(prefix_len=-1), 1), (dict(table_stride=4), 1)]


def append(lib, cache, batch, rot="default", pointers=None, strides=None):
    rot = wb.Rotation(128, 0, 1, (64, 0, 0), 0, 1.0) if rot == "default" else rot
    strides = strides or wb.AppendStrides()
    p = list(range(0x1000, 0x10000, 0x1000))[:11] if pointers is None else pointers
    return lib.waveal_cache_append(ctypes.byref(cache), ctypes.byref(batch), None if rot is None else ctypes.byref(rot), ctypes.byref(strides),
                                   *p, None, None)


@pytest.mark.parametrize("kw, status", BAD_CACHE + [(dict(head_dim=1), 2), (dict(head_dim=600), 2), (dict(head_dim=64), 1)])
def test_append_refuses_cache(lib, kw, status):
    assert append(lib, cache_desc(**kw), batch_desc()) == status


@pytest.mark.parametrize("kw, status", BAD_BATCH + [(dict(q_heads=-1), 1)])
def test_append_refuses_batch(lib, kw, status):
    assert append(lib, cache_desc(), batch_desc(**kw)) == status


def test_append_refuses_pointers(lib):
    good = list(range(0x1000, 0x10000, 0x1000))[:11]
    for i in (0, 1, 2, 3, 4, 5, 6, 7, 8, 10):                         # positions (9) may be left out
        assert append(lib, cache_desc(), batch_desc(), pointers=[None if i == j else p for j, p in enumerate(good)]) == wb.ERR_INVALID_ARG, i
    assert append(lib, cache_desc(), batch_desc(), rot=None) == wb.ERR_INVALID_ARG          # queries, but nothing to turn them by
    assert append(lib, cache_desc(), batch_desc(), pointers=[0x1001] + good[1:]) == wb.ERR_INVALID_ARG
    assert append(lib, cache_desc(), batch_desc(tokens=0), pointers=[None] * 11) == wb.OK
    strides = wb.AppendStrides()
    strides.q[1] = 8
    assert append(lib, cache_desc(), batch_desc(), pointers=good[:3] + [good[2]] + good[4:], strides=strides) == wb.ERR_INVALID_ARG


def attend(lib, cache, batch, pointers=None, q_stride=(128, 512), o_stride=(128, 512), ws=0x100000, ws_bytes=1 << 40):
    p = [0x1000, 0x2000, 0x3000, 0x4000, 0x5000, 0x6000, 0x7000, 0x8000, 0x9000] if pointers is None else pointers
    q, k, v, o, lse, start, lens, table, prefix = p
    return lib.waveal_prefix_attn(ctypes.byref(cache), ctypes.byref(batch), q, (ctypes.c_int64 * 2)(*q_stride), k, v, o,
                                  (ctypes.c_int64 * 2)(*o_stride), lse, start, lens, table, prefix, 0.0, ws, ws_bytes, None, None)


@pytest.mark.parametrize("kw, status", BAD_CACHE + [(dict(head_dim=96), 2), (dict(k_stride=(4096, 2048, 124)), 1), (dict(v_stride=(-4096, 2048, 128)), 1)])
def test_attention_refuses_cache(lib, kw, status):
    assert attend(lib, cache_desc(**kw), batch_desc()) == status
    n = ctypes.c_size_t(0)
    assert lib.waveal_prefix_attn_workspace_bytes(ctypes.byref(cache_desc(**kw)), ctypes.byref(batch_desc()), ctypes.byref(n)) == status


@pytest.mark.parametrize("kw, status", BAD_BATCH + [(dict(q_heads=0), 1), (dict(q_heads=3), 1), (dict(q_heads=258), 1), (dict(flags=2), 1),
                                                    (dict(tokens=1 << 29), 2), (dict(prefix_len=(1 << 30) + 1), 2),
                                                    (dict(max_pages=1 << 27, table_stride=1 << 27), 2)])
def test_attention_refuses_batch(lib, kw, status):
    assert attend(lib, cache_desc(), batch_desc(**kw)) == status


def test_attention_refuses_pointers_strides_workspace(lib):
    good = [0x1000, 0x2000, 0x3000, 0x4000, 0x5000, 0x6000, 0x7000, 0x8000, 0x9000]
    for i in (0, 1, 2, 3, 5, 6, 7, 8):                                # lse (4) may be left out
        assert attend(lib, cache_desc(), batch_desc(), [None if i == j else p for j, p in enumerate(good)]) == wb.ERR_INVALID_ARG, i
    for i in (0, 1, 2, 3):
        assert attend(lib, cache_desc(), batch_desc(), [p + 8 if i == j else p for j, p in enumerate(good)]) == wb.ERR_INVALID_ARG, i
    assert attend(lib, cache_desc(), batch_desc(), q_stride=(128, 516)) == wb.ERR_INVALID_ARG
    assert attend(lib, cache_desc(), batch_desc(), o_stride=(-128, 512)) == wb.ERR_INVALID_ARG
    assert attend(lib, cache_desc(), batch_desc(), ws=None) == wb.ERR_WORKSPACE
    assert attend(lib, cache_desc(), batch_desc(), ws_bytes=1000) == wb.ERR_WORKSPACE
    assert attend(lib, cache_desc(), batch_desc(), ws=0x100010) == wb.ERR_WORKSPACE
    assert attend(lib, cache_desc(), batch_desc(tokens=0), [None] * 9, ws=None) == wb.OK
    n = ctypes.c_size_t(0)
    assert lib.waveal_prefix_attn_workspace_bytes(ctypes.byref(cache_desc()), ctypes.byref(batch_desc()), ctypes.byref(n)) == wb.OK
    assert n.value >= 2 * 3 * 4 * (128 * 4 + 8)
    assert lib.waveal_prefix_attn_workspace_bytes(ctypes.byref(cache_desc()), ctypes.byref(batch_desc()), None) == wb.ERR_INVALID_ARG


def test_binding_checks_types():
    x = torch.zeros((2, 3, 64))
    with pytest.raises(TypeError):
        wb.rope(x, torch.zeros((3,)), torch.zeros((32,)))
    with pytest.raises(ValueError):
        wb.PagedCache(torch.zeros((2, 1, 16, 64)), torch.zeros((2, 1, 16, 64)))
