"""Host-only checks of prompt attention and of the page calls: struct layouts and refusals, all before any CUDA work."""
import ctypes

import pytest
import torch

from paper_2609_34814_b200 import binding as wb
from paper_2609_34814_b200 import build as wbuild


@pytest.fixture(scope="module")
def lib():
    wbuild.build()
    return wb.load()


def test_struct_layouts():
    assert ctypes.sizeof(wb.PromptDesc) == 96 and wb.PromptDesc.q_stride.offset == 32
    assert ctypes.sizeof(wb.ForkDesc) == 32 and ctypes.sizeof(wb.CompactDesc) == 32 and wb.CompactDesc.old_stride.offset == 16
    assert (wb._PROMPT.size, wb._FORK.size, wb._COMPACT.size) == (96, 32, 32)
    d = wb.PromptDesc.from_buffer_copy(wb._PROMPT.pack(*range(1, 16)))
    assert (d.batch, d.tokens, d.q_heads, d.kv_heads, d.head_dim, d.dtype, d.flags, d.q_stride[0], d.o_stride[1]) == (1, 2, 3, 4, 5, 6, 7, 8, 15)
    f = wb.ForkDesc.from_buffer_copy(wb._FORK.pack(1, 2, 3, 4, 5, 6))
    assert (f.old_rows, f.rows, f.old_pages, f.pages, f.old_stride, f.stride) == (1, 2, 3, 4, 5, 6)
    c = wb.CompactDesc.from_buffer_copy(wb._COMPACT.pack(1, 2, 3, 4, 5))
    assert (c.rows, c.pages, c.prefix_pages, c.old_stride, c.stride) == (1, 2, 3, 4, 5)


def prompt(lib, pointers=None, ws=0x100000, ws_bytes=1 << 40, **kw):
    d = wb.PromptDesc(2, 100, 8, 2, 128, wb.BF16, 1, (128, 1024), (128, 256), (128, 256), (128, 1024))
    for k, v in kw.items():
        setattr(d, k, v)
    p = [0x1000, 0x2000, 0x3000, 0x4000, 0x5000, 0x6000, 0x7000] if pointers is None else pointers
    return lib.waveal_prompt_attn(ctypes.byref(d), *p, 0.0, ws, ws_bytes, None, None), d


@pytest.mark.parametrize("kw, status", [
    (dict(batch=-1), 1), (dict(tokens=-1), 1), (dict(q_heads=0), 1), (dict(kv_heads=0), 1), (dict(q_heads=7), 1), (dict(q_heads=258), 1), (dict(head_dim=96), 2),
    (dict(head_dim=256), 2), (dict(dtype=wb.FP32), 2), (dict(dtype=-1), 2), (dict(flags=2), 1), (dict(tokens=1 << 28), 2), (dict(tokens=(1 << 25) + 1), 2), (dict(batch=600_000_000), 2),
    (dict(q_stride=(128, 1020)), 1), (dict(k_stride=(4, 256)), 1), (dict(v_stride=(128, -256)), 1), (dict(o_stride=(130, 1024)), 1)])
def test_prompt_refused(lib, kw, status):
    got, d = prompt(lib, **kw)
    assert got == status and wb.last_error()
    n = ctypes.c_size_t(0)
    assert lib.waveal_prompt_attn_workspace_bytes(ctypes.byref(d), ctypes.byref(n)) == status


def test_prompt_refuses_pointers_and_workspace(lib):
    good = [0x1000, 0x2000, 0x3000, 0x4000, 0x5000, 0x6000, 0x7000]
    for i in (0, 1, 2, 3, 5):                                         # lse (4) and lengths (6) may be left out
        assert prompt(lib, [None if i == j else p for j, p in enumerate(good)])[0] == wb.ERR_INVALID_ARG, i
    for i in range(4):
        assert prompt(lib, [p + 8 if i == j else p for j, p in enumerate(good)])[0] == wb.ERR_INVALID_ARG, i
    for i in range(3):                                                # the results over an input
        assert prompt(lib, [good[i] if j == 3 else p for j, p in enumerate(good)])[0] == wb.ERR_INVALID_ARG, i
    assert prompt(lib, ws=None)[0] == prompt(lib, ws_bytes=100)[0] == prompt(lib, ws=0x100010)[0] == wb.ERR_WORKSPACE
    assert lib.waveal_prompt_attn(None, *good, 0.0, 0x100000, 1 << 40, None, None) == wb.ERR_INVALID_ARG
    assert prompt(lib, [None] * 7, ws=None, tokens=0)[0] == prompt(lib, [None] * 7, ws=None, batch=0)[0] == wb.OK
    n = ctypes.c_size_t(0)
    d = prompt(lib, ws=None)[1]
    assert lib.waveal_prompt_attn_workspace_bytes(ctypes.byref(d), ctypes.byref(n)) == wb.OK and n.value >= 2 * 16
    assert lib.waveal_prompt_attn_workspace_bytes(ctypes.byref(d), None) == wb.ERR_INVALID_ARG


def test_the_stride_of_a_dimension_with_one_entry_is_not_looked_at(lib):
    n = ctypes.c_size_t(0)
    odd = dict(q_stride=(3, -5), k_stride=(1, 1), v_stride=(0, 7), o_stride=(9, 9))
    for kw, status in ((dict(tokens=1, q_heads=1, kv_heads=1, **odd), wb.OK), (dict(tokens=1, q_heads=2, kv_heads=1, **odd), wb.ERR_INVALID_ARG),
                       (dict(tokens=2, q_heads=1, kv_heads=1, **odd), wb.ERR_INVALID_ARG)):
        d = prompt(lib, ws=None, **kw)[1]
        assert lib.waveal_prompt_attn_workspace_bytes(ctypes.byref(d), ctypes.byref(n)) == status


def cache_desc(**kw):
    d = wb.CacheDesc(10, 16, 2, 128, wb.BF16, (4096, 2048, 128), (4096, 2048, 128))
    for k, v in kw.items():
        setattr(d, k, v)
    return d


BAD_CACHE = [(dict(n_pages=0), 1), (dict(kv_heads=0), 1), (dict(page_size=8), 2), (dict(page_size=48), 2), (dict(page_size=1 << 17), 2),
             (dict(kv_heads=1 << 21), 2), (dict(dtype=wb.FP32), 2), (dict(head_dim=1), 2), (dict(head_dim=513), 2),
             (dict(kv_heads=1 << 10, page_size=1 << 15), 2)]
# k, v, old table, held, refs, parents, keep, room, table, new refs
FORK = [0x10000 * i for i in range(1, 11)]


def fork(lib, cache=None, pointers=FORK, ws=0x1000000, ws_bytes=1 << 40, **kw):
    d = wb.ForkDesc(3, 4, 5, 6, 5, 6)
    for k, v in kw.items():
        setattr(d, k, v)
    return lib.waveal_cache_fork(ctypes.byref(cache or cache_desc()), ctypes.byref(d), *pointers, ws, ws_bytes, None, None)


@pytest.mark.parametrize("kw, status", BAD_CACHE)
def test_fork_refuses_cache(lib, kw, status):
    assert fork(lib, cache_desc(**kw)) == status
    n = ctypes.c_size_t(0)
    assert lib.waveal_cache_fork_workspace_bytes(ctypes.byref(cache_desc(**kw)), ctypes.byref(wb.ForkDesc()), ctypes.byref(n)) == status
    assert lib.waveal_cache_compact_workspace_bytes(ctypes.byref(cache_desc(**kw)), ctypes.byref(n)) == status


@pytest.mark.parametrize("kw, status", [(dict(old_rows=-1), 1), (dict(rows=-1), 1), (dict(old_pages=-1), 1), (dict(pages=-1), 1), (dict(old_stride=4), 1),
                                        (dict(stride=5), 1), (dict(rows=1 << 16, pages=1 << 16, stride=1 << 16), 2),
                                        (dict(old_rows=1 << 16, old_pages=1 << 16, old_stride=1 << 16), 2)])
def test_fork_refuses_sizes(lib, kw, status):
    assert fork(lib, **kw) == status


def test_fork_refuses_pointers(lib):
    for i in (0, 1, 2, 3, 4, 6, 7, 8, 9):
        assert fork(lib, pointers=[None if i == j else p for j, p in enumerate(FORK)]) == wb.ERR_INVALID_ARG, i
    assert fork(lib, pointers=FORK[:5] + [None] + FORK[6:]) == wb.ERR_INVALID_ARG           # four rows, but three before
    assert fork(lib, pointers=[FORK[0] + 1] + FORK[1:]) == wb.ERR_INVALID_ARG
    assert fork(lib, pointers=FORK[:8] + [FORK[2] + 40] + FORK[9:]) == wb.ERR_INVALID_ARG   # tables over each other
    assert fork(lib, pointers=FORK[:9] + [FORK[4]]) == wb.ERR_INVALID_ARG                   # counts over each other
    assert fork(lib, ws=None) == fork(lib, ws_bytes=100) == fork(lib, ws=0x1000010) == wb.ERR_WORKSPACE


# k, v, refs, old table, old prefix, new refs, table, prefix, place, used
COMPACT = [0x10000 * i for i in range(1, 11)]


def compact(lib, cache=None, pointers=COMPACT, ws=0x1000000, ws_bytes=1 << 40, **kw):
    d = wb.CompactDesc(3, 5, 2, 5, 5)
    for k, v in kw.items():
        setattr(d, k, v)
    return lib.waveal_cache_compact(ctypes.byref(cache or cache_desc()), ctypes.byref(d), *pointers, ws, ws_bytes, None)


def test_compact_refused(lib):
    for kw, status in BAD_CACHE:
        assert compact(lib, cache_desc(**kw)) == status, kw
    for kw, status in ((dict(rows=-1), 1), (dict(pages=-1), 1), (dict(prefix_pages=-1), 1), (dict(old_stride=4), 1), (dict(stride=4), 1),
                       (dict(rows=1 << 16, pages=1 << 16, old_stride=1 << 16, stride=1 << 16), 2)):
        assert compact(lib, **kw) == status, kw
    for i in range(10):
        assert compact(lib, pointers=[None if i == j else p for j, p in enumerate(COMPACT)]) == wb.ERR_INVALID_ARG, i
    for i, j in ((5, 2), (6, 3), (7, 4)):
        assert compact(lib, pointers=[COMPACT[j] + 4 if n == i else p for n, p in enumerate(COMPACT)]) == wb.ERR_INVALID_ARG
    assert compact(lib, ws=None) == compact(lib, ws_bytes=10) == compact(lib, ws=0x1000004) == wb.ERR_WORKSPACE


def test_copy_refused(lib):
    def copy(to=None, source=None, count=3, pointers=(0x1000, 0x2000, 0x3000, 0x4000, 0x5000, 0x6000)):
        return lib.waveal_cache_copy(ctypes.byref(to or cache_desc()), ctypes.byref(source or cache_desc()), count, *pointers, None, None)
    for kw, status in BAD_CACHE:
        assert copy(cache_desc(**kw)) == copy(source=cache_desc(**kw)) == status, kw
    for kw in (dict(page_size=32), dict(kv_heads=3), dict(head_dim=64), dict(dtype=wb.FP16)):
        assert copy(cache_desc(**kw)) == wb.ERR_INVALID_ARG, kw
    assert copy(count=-1) == wb.ERR_INVALID_ARG
    good = [0x1000, 0x2000, 0x3000, 0x4000, 0x5000, 0x6000]
    for i in range(6):
        assert copy(pointers=[None if i == j else p for j, p in enumerate(good)]) == wb.ERR_INVALID_ARG, i
    assert copy(count=0, pointers=[None] * 6) == wb.OK


def test_status_text(lib):
    assert "pages" in wb.status_string(wb.ERR_NO_PAGES)


def test_binding_checks_types():
    x = torch.zeros((2, 3, 64))
    with pytest.raises((TypeError, ValueError)):
        wb.prompt_attn(x, x, x, torch.zeros((2,), dtype=torch.int32))
    with pytest.raises(ValueError):
        wb.PagedCache(torch.zeros((2, 1, 16, 64)), torch.zeros((2, 1, 16, 64)))
