"""ctypes binding of libwaveal.so: the same names as include/waveal.h, argument marshalling only.

Every step of the hot path runs inside the library's CUDA kernels; this module converts
torch tensors to pointers, allocates the workspaces the C ABI asks the caller to own, and
raises on a non-zero status.  It fails loudly when the library is missing: there is no CPU
fallback.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import NamedTuple, Optional

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libwaveal.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_BAD_MASK, ERR_CUDA, ERR_TIMEOUT, ERR_NO_PAGES = range(8)
AUTO, FORCE_REORDER, FORCE_NATURAL, STAGE1_ONLY, STAGE2_ONLY = range(5)
FLAG_SKIPPED, FLAG_SHORT_SEQ, FLAG_TOO_SPARSE, FLAG_ALREADY_LOCAL = 1, 2, 4, 8

EXPORTS = ["waveal_plan_desc_default", "waveal_plan_workspace_bytes", "waveal_plan_bitmap", "waveal_plan_csr",
           "waveal_bitmap_to_csr", "waveal_bitmap_to_csr_noalloc", "waveal_noalloc_max_rows",
           "waveal_gather_rows", "waveal_scatter_rows", "waveal_bsattn_workspace_bytes", "waveal_bsattn_fwd",
           "waveal_rope_freqs", "waveal_rope", "waveal_cache_append", "waveal_prefix_attn_workspace_bytes", "waveal_prefix_attn",
           "waveal_prompt_attn_workspace_bytes", "waveal_prompt_attn", "waveal_cache_fork_workspace_bytes", "waveal_cache_fork",
           "waveal_cache_compact_workspace_bytes", "waveal_cache_compact", "waveal_cache_copy",
           "waveal_default_wave_size", "waveal_last_launch_count", "waveal_status_string", "waveal_last_error"]


class PlanDesc(ctypes.Structure):
    _fields_ = [("heads", ctypes.c_int32), ("n_q_blocks", ctypes.c_int32), ("n_kv_blocks", ctypes.c_int32),
                ("wave_size", ctypes.c_int32), ("svd_iters", ctypes.c_int32), ("mode", ctypes.c_int32),
                ("seed", ctypes.c_uint64), ("kv_bytes_per_head", ctypes.c_int64), ("l2_bytes", ctypes.c_int64),
                ("l2_fit_num", ctypes.c_int32), ("l2_fit_den", ctypes.c_int32), ("min_density_ppm", ctypes.c_int32),
                ("local_num", ctypes.c_int32), ("local_den", ctypes.c_int32), ("min_nnz", ctypes.c_int64)]


class PlanOut(ctypes.Structure):
    _fields_ = [("row_order", ctypes.c_void_p), ("row_nnz", ctypes.c_void_p), ("skip_flags", ctypes.c_void_p),
                ("col_count", ctypes.c_void_p), ("order1", ctypes.c_void_p), ("embedding", ctypes.c_void_p),
                ("stats", ctypes.c_void_p), ("dev_status", ctypes.c_void_p)]


class AttnDesc(ctypes.Structure):
    _fields_ = [("heads", ctypes.c_int32), ("seq_q", ctypes.c_int32), ("seq_kv", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("block_q", ctypes.c_int32), ("block_kv", ctypes.c_int32),
                ("q_stride", ctypes.c_int64 * 2), ("k_stride", ctypes.c_int64 * 2), ("v_stride", ctypes.c_int64 * 2),
                ("o_stride", ctypes.c_int64 * 2), ("order_heads_interleaved", ctypes.c_int32),
                ("flags", ctypes.c_int32)]


class Rotation(ctypes.Structure):
    _fields_ = [("rot_dim", ctypes.c_int32), ("pairs", ctypes.c_int32), ("axes", ctypes.c_int32),
                ("axis_pairs", ctypes.c_int32 * 3), ("inverse", ctypes.c_int32), ("amplitude", ctypes.c_float)]


class RopeDesc(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("q_heads", ctypes.c_int32),
                ("k_heads", ctypes.c_int32), ("dtype", ctypes.c_int32), ("rot", Rotation),
                ("q_stride", ctypes.c_int64 * 2), ("q_out_stride", ctypes.c_int64 * 2),
                ("k_stride", ctypes.c_int64 * 2), ("k_out_stride", ctypes.c_int64 * 2)]


class CacheDesc(ctypes.Structure):
    _fields_ = [("n_pages", ctypes.c_int32), ("page_size", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32), ("k_stride", ctypes.c_int64 * 3),
                ("v_stride", ctypes.c_int64 * 3)]


class BatchDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("tokens", ctypes.c_int32), ("q_heads", ctypes.c_int32),
                ("max_pages", ctypes.c_int32), ("prefix_len", ctypes.c_int32), ("flags", ctypes.c_int32),
                ("table_stride", ctypes.c_int64)]


class AppendStrides(ctypes.Structure):
    _fields_ = [("k", ctypes.c_int64 * 2), ("v", ctypes.c_int64 * 2), ("q", ctypes.c_int64 * 2),
                ("q_out", ctypes.c_int64 * 2)]


class PromptDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("tokens", ctypes.c_int32), ("q_heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32), ("flags", ctypes.c_int32), ("q_stride", ctypes.c_int64 * 2),
                ("k_stride", ctypes.c_int64 * 2), ("v_stride", ctypes.c_int64 * 2), ("o_stride", ctypes.c_int64 * 2)]


class ForkDesc(ctypes.Structure):
    _fields_ = [("old_rows", ctypes.c_int32), ("rows", ctypes.c_int32), ("old_pages", ctypes.c_int32), ("pages", ctypes.c_int32),
                ("old_stride", ctypes.c_int64), ("stride", ctypes.c_int64)]


class CompactDesc(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int32), ("pages", ctypes.c_int32), ("prefix_pages", ctypes.c_int32), ("old_stride", ctypes.c_int64),
                ("stride", ctypes.c_int64)]


class WavealError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"waveal status {status}: {message}")
        self.status = status


_lib = None


def load() -> ctypes.CDLL:
    """Loads the C-ABI library; raises if it was not built (no fallback exists)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: run `python -m paper_2609_34814_b200.build` "
                               "(the library has no CPU fallback)")
        lib = ctypes.CDLL(LIB_PATH)
        P, I32, I64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
        lib.waveal_plan_desc_default.argtypes = [ctypes.POINTER(PlanDesc)]
        lib.waveal_plan_desc_default.restype = None
        lib.waveal_plan_workspace_bytes.argtypes = [ctypes.POINTER(PlanDesc), ctypes.POINTER(ctypes.c_size_t)]
        lib.waveal_plan_bitmap.argtypes = [ctypes.POINTER(PlanDesc), P, P, ctypes.c_size_t, ctypes.POINTER(PlanOut), P]
        lib.waveal_plan_csr.argtypes = [ctypes.POINTER(PlanDesc), P, P, P, ctypes.c_size_t, ctypes.POINTER(PlanOut), P]
        lib.waveal_bitmap_to_csr.argtypes = [I32, I32, I32, P, P, P, I64, P, ctypes.c_size_t, P]
        lib.waveal_bitmap_to_csr_noalloc.argtypes = [I32, I32, I32, P, P, P, I64, P]
        lib.waveal_bitmap_to_csr_noalloc.restype = ctypes.c_int
        lib.waveal_noalloc_max_rows.restype = ctypes.c_size_t
        for name in ("waveal_gather_rows", "waveal_scatter_rows"):
            getattr(lib, name).argtypes = [I32, I32, I32, I32, P, ctypes.POINTER(I64), P, ctypes.POINTER(I64), P, P]
            getattr(lib, name).restype = ctypes.c_int
        lib.waveal_bsattn_workspace_bytes.argtypes = [ctypes.POINTER(AttnDesc), ctypes.POINTER(ctypes.c_size_t)]
        lib.waveal_bsattn_fwd.argtypes = [ctypes.POINTER(AttnDesc), P, P, P, P, P, P, P, P, ctypes.c_float, P,
                                          ctypes.c_size_t, P, P]
        lib.waveal_rope_freqs.argtypes = [I32, ctypes.c_double, ctypes.c_int, ctypes.c_double, I64, P, ctypes.POINTER(ctypes.c_float)]
        # (the descriptors of these come as packed bytes: half the host's time of structures filled field by field)
        lib.waveal_rope.argtypes = [P] * 8
        lib.waveal_cache_append.argtypes = [P] * 17
        lib.waveal_prefix_attn_workspace_bytes.argtypes = [P, P, ctypes.POINTER(ctypes.c_size_t)]
        lib.waveal_prefix_attn.argtypes = [P] * 13 + [ctypes.c_float, P, ctypes.c_size_t, P, P]
        lib.waveal_prompt_attn_workspace_bytes.argtypes = [P, ctypes.POINTER(ctypes.c_size_t)]
        lib.waveal_prompt_attn.argtypes = [P] * 8 + [ctypes.c_float, P, ctypes.c_size_t, P, P]
        lib.waveal_cache_fork_workspace_bytes.argtypes = [P, P, ctypes.POINTER(ctypes.c_size_t)]
        lib.waveal_cache_fork.argtypes = [P] * 13 + [ctypes.c_size_t, P, P]
        lib.waveal_cache_compact_workspace_bytes.argtypes = [P, ctypes.POINTER(ctypes.c_size_t)]
        lib.waveal_cache_compact.argtypes = [P] * 13 + [ctypes.c_size_t, P]
        lib.waveal_cache_copy.argtypes = [P, P, I32] + [P] * 8
        for name in ["waveal_prompt_attn_workspace_bytes", "waveal_prompt_attn", "waveal_cache_fork_workspace_bytes", "waveal_cache_fork",
                     "waveal_cache_compact_workspace_bytes", "waveal_cache_compact", "waveal_cache_copy",
                     "waveal_rope_freqs", "waveal_rope", "waveal_cache_append", "waveal_prefix_attn_workspace_bytes", "waveal_prefix_attn",
                     "waveal_plan_workspace_bytes", "waveal_plan_bitmap", "waveal_plan_csr", "waveal_bitmap_to_csr",
                     "waveal_gather_rows", "waveal_scatter_rows", "waveal_bsattn_workspace_bytes", "waveal_bsattn_fwd", "waveal_default_wave_size",
                     "waveal_last_launch_count"]:
            getattr(lib, name).restype = ctypes.c_int
        lib.waveal_status_string.argtypes = [ctypes.c_int]
        lib.waveal_status_string.restype = ctypes.c_char_p
        lib.waveal_last_error.restype = ctypes.c_char_p
        _lib = lib
    return _lib


def last_error() -> str:
    return load().waveal_last_error().decode()


def status_string(s: int) -> str:
    return load().waveal_status_string(s).decode()


def _check(status: int):
    if status != OK:
        raise WavealError(status, last_error() or status_string(status))


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:
        import torch
        # the handle of the current stream without a Stream object around it (3.3 us each, three times a step)
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice()) or None
    return stream.cuda_stream or None


def default_wave_size() -> int:
    return int(load().waveal_default_wave_size())


def last_launch_count() -> int:
    return int(load().waveal_last_launch_count())


def plan_desc_default(**kw) -> PlanDesc:
    d = PlanDesc()
    load().waveal_plan_desc_default(ctypes.byref(d))
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def plan_workspace_bytes(desc: PlanDesc) -> int:
    n = ctypes.c_size_t(0)
    _check(load().waveal_plan_workspace_bytes(ctypes.byref(desc), ctypes.byref(n)))
    return int(n.value)


class PlanResult:
    """Device tensors a plan call filled (torch tensors; the caller may pass its own)."""

    def __init__(self, **kw):
        self.__dict__.update(kw)

    def __getattr__(self, name):
        # the status words, cleared by the call: a view of them is made for those who look (1.8 us of the smallest step's 41)
        if name != "dev_status" or "_words" not in self.__dict__:
            raise AttributeError(name)
        buf, at = self._words
        self.dev_status = buf.as_strided((4,), (1,), at)
        return self.dev_status


def _plan_outputs(desc: PlanDesc, like, debug: bool):
    import torch
    H, M, N = desc.heads, desc.n_q_blocks, desc.n_kv_blocks
    device = like.device
    # one allocation: a tensor per output took more of the host's time than the call itself
    at_flags, at_status = 2 * H * M, 2 * H * M + (H + 3) // 4
    buf = like.new_empty((at_status + 4,), dtype=torch.int32)
    res = PlanResult(
        row_order=buf.as_strided((H, M), (M, 1), 0),
        row_nnz=buf.as_strided((H, M), (M, 1), H * M),
        skip_flags=buf.view(torch.uint8).as_strided((H,), (1,), 4 * at_flags),
        _words=(buf, at_status),
        col_count=None, order1=None, embedding=None, stats=None)
    if debug:
        res.col_count = torch.empty((H, N), dtype=torch.int32, device=device)
        res.order1 = torch.empty((H, M), dtype=torch.int32, device=device)
        res.embedding = torch.empty((H, M, 2), dtype=torch.float64, device=device)
        res.stats = torch.empty((H, 4), dtype=torch.int64, device=device)
    out = PlanOut(_ptr(res.row_order), _ptr(res.row_nnz), _ptr(res.skip_flags), _ptr(res.col_count),
                  _ptr(res.order1), _ptr(res.embedding), _ptr(res.stats), buf.data_ptr() + 4 * at_status)
    return res, out


def plan_bitmap(desc: PlanDesc, mask_bits, workspace=None, debug: bool = False, stream=None) -> PlanResult:
    """waveal_plan_bitmap.  mask_bits: cuda tensor of 64-bit words [heads, M_B, ceil(N_B/64)].  A bitmap holds
    nothing that could be malformed: the result's dev_status is zero (cleared by the call's first kernel: a launch
    of its own for four words took 7 of the smallest step's 47 us)."""
    import torch
    lib = load()
    if workspace is None:
        workspace = torch.empty((plan_workspace_bytes(desc) + 256,), dtype=torch.uint8, device=mask_bits.device)
    res, out = _plan_outputs(desc, mask_bits, debug)
    res.workspace = workspace
    own = PlanDesc.from_buffer_copy(desc)            # (the caller's may serve several threads)
    own.mode |= PLAN_CLEAR_STATUS
    _check(lib.waveal_plan_bitmap(ctypes.byref(own), _ptr(mask_bits), _ptr(workspace), workspace.numel(),
                                  ctypes.byref(out), _stream(stream)))
    return res


def plan_csr(desc: PlanDesc, kv_row_ptr, kv_block_indices, workspace=None, debug: bool = False, stream=None) -> PlanResult:
    """waveal_plan_csr.  dev_status reports an index out of range."""
    import torch
    lib = load()
    if workspace is None:
        workspace = torch.empty((plan_workspace_bytes(desc) + 256,), dtype=torch.uint8, device=kv_row_ptr.device)
    res, out = _plan_outputs(desc, kv_row_ptr, debug)
    res.workspace = workspace
    # cleared on the call's own stream: ordered before the kernels that may report something
    if stream is None:
        res.dev_status.zero_()
    else:
        own = stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(stream.cuda_stream, kv_row_ptr.device)
        with torch.cuda.stream(own):
            res.dev_status.zero_()
    _check(lib.waveal_plan_csr(ctypes.byref(desc), _ptr(kv_row_ptr), _ptr(kv_block_indices), _ptr(workspace),
                               workspace.numel(), ctypes.byref(out), _stream(stream)))
    return res


def bitmap_to_csr(mask_bits, n_kv_blocks: int, capacity: Optional[int] = None, stream=None):
    """waveal_bitmap_to_csr.  Returns (kv_row_ptr, kv_block_indices) device tensors; when
    `capacity` is None the row pointers are computed first and their last entry read back
    (one synchronisation) to size the index array."""
    import torch
    lib = load()
    H, M, _ = mask_bits.shape
    n = H * M + 1
    if capacity is None:
        buf = mask_bits.new_empty((2 * n,), dtype=torch.int32)
        at = buf.data_ptr()
        _check(lib.waveal_bitmap_to_csr(H, M, n_kv_blocks, _ptr(mask_bits), at, None, 0, at + 4 * n, 4 * n, _stream(stream)))
        capacity = int(buf[n - 1].item())
    # the call's workspace behind the row pointers; the indices by themselves: a caller that keeps the row
    # pointers alone does not keep the lists
    buf = mask_bits.new_empty((2 * n,), dtype=torch.int32)
    idx = mask_bits.new_empty((max(capacity, 1),), dtype=torch.int32)
    at = buf.data_ptr()
    _check(lib.waveal_bitmap_to_csr(H, M, n_kv_blocks, _ptr(mask_bits), at, idx.data_ptr(), capacity, at + 4 * n, 4 * n,
                                    _stream(stream)))
    return buf.as_strided((n,), (1,), 0), idx if capacity > 0 else idx[:0]


def noalloc_max_rows() -> int:
    return int(load().waveal_noalloc_max_rows())


def bitmap_to_csr_noalloc(mask_bits, n_kv_blocks: int, kv_row_ptr, kv_block_indices, stream=None):
    """waveal_bitmap_to_csr_noalloc: for callers that cannot allocate device memory (an engine
    plug-in handed pre-planned tensors).  Every buffer is the caller's: `kv_row_ptr` int32
    [heads*M_B + 1] and `kv_block_indices` int32 [capacity] (or None for row pointers only)
    are filled on the stream; the call itself allocates nothing, here or in the library, and
    refuses problems with more than noalloc_max_rows() query-block rows."""
    H, M, _ = mask_bits.shape
    cap = 0 if kv_block_indices is None else kv_block_indices.numel()
    _check(load().waveal_bitmap_to_csr_noalloc(H, M, n_kv_blocks, _ptr(mask_bits), _ptr(kv_row_ptr),
                                               _ptr(kv_block_indices), cap, _stream(stream)))


def _move_rows(fn_name: str, src, dst, row_order, block: int, stream=None):
    """src, dst: [heads, n_blocks*block, row elements] tensors (last dim contiguous)."""
    H, rows, _ = src.shape
    assert src.stride(2) == 1 and dst.stride(2) == 1 and dst.shape == src.shape
    es = src.element_size()
    ss = (ctypes.c_int64 * 2)(src.stride(0) * es, src.stride(1) * es)
    ds = (ctypes.c_int64 * 2)(dst.stride(0) * es, dst.stride(1) * es)
    _check(getattr(load(), fn_name)(H, rows // block, block, src.shape[2] * es, _ptr(src), ss, _ptr(dst), ds,
                                    _ptr(row_order), _stream(stream)))


def gather_rows(src, dst, row_order, block: int, stream=None):
    """waveal_gather_rows: dst block p <- src block row_order[h][p]."""
    _move_rows("waveal_gather_rows", src, dst, row_order, block, stream)


def scatter_rows(src, dst, row_order, block: int, stream=None):
    """waveal_scatter_rows: dst block row_order[h][p] <- src block p."""
    _move_rows("waveal_scatter_rows", src, dst, row_order, block, stream)


RING_CUT_LARGEST_GAP = 16
PLAN_CLEAR_STATUS = 32
ATTN_ONLINE_MAX_ONLY = 1
ATTN_SELFTEST_LOST_TILE = 256
ATTN_NO_ROW_PAIRING = 2


def attn_desc(q, k, v, o, seq_q: int, seq_kv: int, block: int, interleaved: bool = False, flags: int = 0) -> AttnDesc:
    """Descriptor for [heads, tokens, head_dim] tensors (head_dim contiguous)."""
    d = AttnDesc()
    d.heads, d.seq_q, d.seq_kv, d.head_dim = q.shape[0], seq_q, seq_kv, q.shape[2]
    d.block_q = d.block_kv = block
    for name, t in (("q_stride", q), ("k_stride", k), ("v_stride", v), ("o_stride", o)):
        assert t.stride(2) == 1, "head_dim must be contiguous"
        getattr(d, name)[0], getattr(d, name)[1] = t.stride(0), t.stride(1)
    d.order_heads_interleaved = 1 if interleaved else 0
    d.flags = flags
    return d


def bsattn_workspace_bytes(desc: AttnDesc) -> int:
    n = ctypes.c_size_t(0)
    _check(load().waveal_bsattn_workspace_bytes(ctypes.byref(desc), ctypes.byref(n)))
    return int(n.value)


def bsattn_fwd(desc: AttnDesc, q, k, v, o, kv_row_ptr, kv_block_indices, row_order=None, lse=None,
               scale: float = 0.0, workspace=None, dev_status=None, stream=None):
    """waveal_bsattn_fwd.  All tensors are cuda tensors owned by the caller; returns nothing
    (o, lse and dev_status are written on the stream)."""
    import torch
    lib = load()
    if workspace is None:
        workspace = torch.empty((bsattn_workspace_bytes(desc),), dtype=torch.uint8, device=q.device)
    _check(lib.waveal_bsattn_fwd(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), _ptr(kv_row_ptr),
                                 _ptr(kv_block_indices), _ptr(row_order), ctypes.c_float(scale), _ptr(workspace),
                                 workspace.numel(), _ptr(dev_status), _stream(stream)))
    return workspace


# ------------------------------------------------------------------ rotary positions, paged cache, shared prefix

BF16, FP16, FP32 = range(3)
PAIRS_HALVES, PAIRS_INTERLEAVED = range(2)
ROPE_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "parts": 3}
PREFIX_CAUSAL = 1
PREFIX_SELFTEST_LOST_TILE = 256


_torch = None
_dtypes = {}


def _load_torch():
    global _torch
    if _torch is None:
        import torch
        _dtypes.update({torch.bfloat16: BF16, torch.float16: FP16, torch.float32: FP32})
        _torch = torch
    return _torch


# waveal_rotation, waveal_rope_desc, waveal_cache_desc, waveal_batch_desc, waveal_append_strides as the C compiler lays them out
_ROTATION = struct.Struct("iii3iif")
_ROPE = struct.Struct("5i" + "iii3iif" + "8q")
_CACHE = struct.Struct("5i6q")
_BATCH = struct.Struct("6iq")
_STRIDES = struct.Struct("8q")
_PAIR = struct.Struct("2q")


def _dtype(t) -> int:
    d = _dtypes.get(t.dtype)
    if d is None:
        raise TypeError(f"{t.dtype} is not supported")
    return d


def rope_freqs(rot_dim: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0, trained_len: int = 0, device="cuda"):
    """waveal_rope_freqs.  Returns (freqs, amplitude): an int64 tensor of rot_dim/2 phase steps on `device` and the
    factor that the scaling puts on the rotated channels.  Several axes: one call each, torch.cat of the steps."""
    torch = _load_torch()
    freqs = torch.empty((rot_dim // 2,), dtype=torch.int64)
    amplitude = ctypes.c_float(1.0)
    _check(load().waveal_rope_freqs(rot_dim, base, ROPE_SCALINGS[scaling], factor, trained_len, freqs.data_ptr(),
                                    ctypes.byref(amplitude)))
    return freqs.to(device), float(amplitude.value)


def _rotation(freqs, interleaved, axis_pairs, amplitude, inverse=False):
    """the numbers of a waveal_rotation"""
    if freqs.dtype is not _torch.int64 or not freqs.is_cuda or freqs.dim() != 1 or not freqs.is_contiguous():
        raise TypeError("freqs must be a contiguous int64 cuda tensor [rot_dim/2]")
    pairs = freqs.shape[0]
    if axis_pairs is None:
        return 2 * pairs, 1 if interleaved else 0, 1, pairs, 0, 0, 1 if inverse else 0, amplitude
    n = len(axis_pairs)
    if n > 3:
        raise ValueError("at most three axes")
    return (2 * pairs, 1 if interleaved else 0, n, axis_pairs[0], axis_pairs[1] if n > 1 else 0, axis_pairs[2] if n > 2 else 0,
            1 if inverse else 0, amplitude)


def _rows(name, t):
    """strides of a [heads, tokens, head_dim] cuda tensor"""
    st = t.stride()
    if len(st) != 3 or not t.is_cuda:
        raise ValueError(f"{name} must be a [heads, tokens, head_dim] cuda tensor")
    if st[2] != 1 and t.shape[2] > 1:
        raise ValueError(f"{name}: head_dim must be contiguous")
    return st


def _new(stream, make):
    """make(), its memory belonging to the call's stream: a block of the current stream's could still be in use there, or be
    handed on there before the call has run"""
    if stream is None:
        return make()
    own = stream if isinstance(stream, _torch.cuda.Stream) else _torch.cuda.ExternalStream(stream.cuda_stream)
    with _torch.cuda.stream(own):
        return make()


def _output(name, out, like, stream):
    """a new tensor like `like`, or the caller's"""
    if out is None:
        return _torch.empty_like(like) if stream is None else _new(stream, lambda: _torch.empty_like(like))
    if out.shape != like.shape or out.dtype is not like.dtype:
        raise ValueError(f"{name} must have its input's shape and type")
    return out


def _status(dev_status):
    if dev_status is None:
        return None
    if dev_status.dtype is not _torch.int32 or not dev_status.is_cuda:
        raise TypeError("dev_status must be an int32 cuda tensor")
    if dev_status.numel() < 4 or not dev_status.is_contiguous():
        raise ValueError("dev_status must be four contiguous words")
    return dev_status.data_ptr()


def _positions(positions, axes, tokens):
    if positions.dtype is not _torch.int32 or not positions.is_cuda:
        raise TypeError("positions must be an int32 cuda tensor")
    shape = positions.shape
    if not (shape == (axes, tokens) or (axes == 1 and shape == (tokens,))) or not positions.is_contiguous():
        raise ValueError(f"positions must be contiguous [{axes}, {tokens}], got {tuple(shape)}")
    return positions.data_ptr()


def rope(q, positions, freqs, k=None, q_out=None, k_out=None, interleaved: bool = False, axis_pairs=None, amplitude: float = 1.0,
         inverse: bool = False, stream=None):
    """waveal_rope.  q (and k): [heads, tokens, head_dim] cuda tensors, head_dim contiguous, any other strides (a
    [tokens, heads, head_dim] tensor is passed as x.transpose(0, 1)); positions: int32 [axes, tokens] ([tokens] for one axis);
    freqs: from rope_freqs.  Returns (q_out, k_out): new tensors unless given (q_out=q turns in place).  inverse=True is the
    gradient: pass those of the outputs, get those of the inputs."""
    _load_torch()
    rot = _rotation(freqs, interleaved, axis_pairs, amplitude, inverse)
    q_st = _rows("q", q)
    heads, tokens, dim = q.shape
    at = _positions(positions, rot[2], tokens)
    q_out = _output("q_out", q_out, q, stream)
    qo_st = _rows("q_out", q_out)
    if k is None:
        k_heads, k_ptr, ko_ptr, k_st, ko_st, k_out = 0, None, None, (0, 0), (0, 0), None
    else:
        k_st = _rows("k", k)
        k_heads = k.shape[0]
        if k.shape[1] != tokens or k.shape[2] != dim or k.dtype is not q.dtype:
            raise ValueError("k must have q's tokens, head_dim and type")
        k_out = _output("k_out", k_out, k, stream)
        ko_st = _rows("k_out", k_out)
        k_ptr, ko_ptr = k.data_ptr(), k_out.data_ptr()
    desc = _ROPE.pack(tokens, dim, heads, k_heads, _dtype(q), *rot, q_st[0], q_st[1], qo_st[0], qo_st[1], k_st[0], k_st[1], ko_st[0], ko_st[1])
    _check(load().waveal_rope(desc, q.data_ptr(), q_out.data_ptr(), k_ptr, ko_ptr, at, freqs.data_ptr(), _stream(stream)))
    return q_out, k_out


class PagedCache:
    """A paged cache of the caller's tensors: k, v [n_pages, kv_heads, page_size, head_dim], bf16 or fp16, head_dim
    contiguous, any other strides ([n_pages, page_size, kv_heads, head_dim] tensors are passed as x.transpose(1, 2))."""

    def __init__(self, k, v):
        _load_torch()
        shape, ks, vs = k.shape, k.stride(), v.stride()
        if len(ks) != 4 or shape != v.shape or k.dtype is not v.dtype or not (k.is_cuda and v.is_cuda):
            raise ValueError("k and v must be cuda tensors [n_pages, kv_heads, page_size, head_dim] of one shape and type")
        if ks[3] != 1 or vs[3] != 1:
            raise ValueError("head_dim must be contiguous")
        self.k, self.v, self.dtype = k, v, k.dtype
        self.n_pages, self.kv_heads, self.page_size, self.head_dim = shape
        self.desc = _CACHE.pack(shape[0], shape[2], shape[1], shape[3], _dtype(k), ks[0], ks[1], ks[2], vs[0], vs[1], vs[2])


def batch_desc(q_heads: int, tokens: int, seq_start, kv_len, page_table=None, prefix_len: int = 0, flags: int = 0) -> bytes:
    """The waveal_batch_desc of a call, from its tensors."""
    int32 = _load_torch().int32
    batch = kv_len.shape[0]
    if kv_len.dtype is not int32 or seq_start.dtype is not int32 or not (kv_len.is_cuda and seq_start.is_cuda):
        raise TypeError("seq_start and kv_len must be int32 cuda tensors")
    if seq_start.shape != (batch + 1,) or kv_len.dim() != 1 or not (seq_start.is_contiguous() and kv_len.is_contiguous()):
        raise ValueError("seq_start must be a contiguous [batch + 1], kv_len a contiguous [batch]")
    if page_table is None:
        return _BATCH.pack(batch, tokens, q_heads, 0, prefix_len, flags, 0)
    if page_table.dtype is not int32 or not page_table.is_cuda:
        raise TypeError("page_table must be an int32 cuda tensor")
    pages, st = page_table.shape, page_table.stride()
    if len(st) != 2 or pages[0] != batch or st[1] != 1 and pages[1] > 1:
        raise ValueError("page_table must be [batch, pages], a row's pages contiguous")
    return _BATCH.pack(batch, tokens, q_heads, pages[1], prefix_len, flags, st[0] if batch > 1 else max(st[0], pages[1]))


def cache_append(cache: PagedCache, k, v, seq_start, kv_len, page_table, positions=None, freqs=None, q=None, q_out=None,
                 prefix_len: int = 0, interleaved: bool = False, axis_pairs=None, amplitude: float = 1.0, dev_status=None, stream=None):
    """waveal_cache_append.  k, v: [kv_heads, tokens, head_dim] of the new tokens; kv_len counts them in.  With freqs the keys
    are rotated on the way (positions None: prefix_len + place among the sequence's own keys), and q [q_heads, tokens, head_dim],
    where given, into q_out (a new tensor unless given; q_out=q turns in place), which is returned."""
    _load_torch()
    k_st, v_st = _rows("k", k), _rows("v", v)
    shape = k.shape
    heads, tokens, dim = shape
    if v.shape != shape or heads != cache.kv_heads or dim != cache.head_dim:
        raise ValueError("k and v must be [kv_heads, tokens, head_dim] of the cache")
    if k.dtype is not cache.dtype or v.dtype is not cache.dtype:
        raise TypeError("k and v must have the cache's type")
    rot = freqs_ptr = at = q_ptr = qo_ptr = None
    if freqs is not None:
        numbers = _rotation(freqs, interleaved, axis_pairs, amplitude)
        rot, freqs_ptr = _ROTATION.pack(*numbers), freqs.data_ptr()
        if positions is not None:
            at = _positions(positions, numbers[2], tokens)
    q_heads, q_st, qo_st = 0, (0, 0), (0, 0)
    if q is not None:
        q_st = _rows("q", q)
        q_heads = q.shape[0]
        if q.shape[1] != tokens or q.shape[2] != dim or q.dtype is not k.dtype:
            raise ValueError("q must have k's tokens, head_dim and type")
        q_out = _output("q_out", q_out, q, stream)
        qo_st = _rows("q_out", q_out)
        q_ptr, qo_ptr = q.data_ptr(), q_out.data_ptr()
    batch = batch_desc(q_heads, tokens, seq_start, kv_len, page_table, prefix_len)
    strides = _STRIDES.pack(k_st[0], k_st[1], v_st[0], v_st[1], q_st[0], q_st[1], qo_st[0], qo_st[1])
    _check(load().waveal_cache_append(cache.desc, batch, rot, strides, k.data_ptr(), v.data_ptr(), q_ptr, qo_ptr, cache.k.data_ptr(),
                                      cache.v.data_ptr(), seq_start.data_ptr(), kv_len.data_ptr(), _ptr(page_table), at, freqs_ptr,
                                      _status(dev_status), _stream(stream)))
    return q_out


def prefix_attn_workspace_bytes(cache: PagedCache, batch: bytes) -> int:
    """Bytes for prefix_attn's workspace; batch: batch_desc of the call."""
    n = ctypes.c_size_t(0)
    _check(load().waveal_prefix_attn_workspace_bytes(cache.desc, batch, ctypes.byref(n)))
    return n.value


def prefix_attn(cache: PagedCache, q, seq_start, kv_len, page_table=None, prefix_pages=None, prefix_len: int = 0, o=None, lse=None,
                return_lse: bool = False, causal: bool = True, scale: float = 0.0, workspace=None, dev_status=None, flags: int = 0, stream=None):
    """waveal_prefix_attn.  q: [q_heads, tokens, head_dim], the new tokens of all sequences one after another; prefix_pages:
    int32 pages of the first prefix_len keys, seen by all; page_table int32 [batch, pages] and kv_len: each sequence's
    own keys, its new ones last.  Returns o (laid out like q unless given), or (o, lse) with return_lse.  What the call allocates belongs
    to its stream."""
    torch = _load_torch()
    q_st = _rows("q", q)
    heads, tokens, dim = q.shape
    if q.dtype is not cache.dtype:
        raise TypeError("q must have the cache's type")
    if dim != cache.head_dim:
        raise ValueError(f"q has head_dim {dim}, the cache {cache.head_dim}")
    batch = batch_desc(heads, tokens, seq_start, kv_len, page_table, prefix_len, (PREFIX_CAUSAL if causal else 0) | flags)
    prefix_ptr = None
    if prefix_pages is not None:
        if prefix_pages.dtype is not torch.int32 or not prefix_pages.is_cuda:
            raise TypeError("prefix_pages must be an int32 cuda tensor")
        if prefix_pages.dim() != 1 or not prefix_pages.is_contiguous() or prefix_pages.shape[0] * cache.page_size < prefix_len:
            raise ValueError("prefix_pages must be a contiguous list of all of the prefix's pages")
        prefix_ptr = prefix_pages.data_ptr()
    o = _output("o", o, q, stream)
    o_st = _rows("o", o)
    if lse is None:
        if return_lse:
            lse = _new(stream, lambda: q.new_empty((heads, tokens), dtype=torch.float32))
    elif lse.dtype is not torch.float32 or lse.shape != (heads, tokens) or not lse.is_cuda or not lse.is_contiguous():
        raise ValueError("lse must be a contiguous float32 cuda tensor [q_heads, tokens]")
    if workspace is None:
        workspace = _new(stream, lambda: q.new_empty((prefix_attn_workspace_bytes(cache, batch),), dtype=torch.uint8))
    elif workspace.dtype is not torch.uint8 or not workspace.is_cuda or not workspace.is_contiguous():
        raise TypeError("workspace must be a contiguous uint8 cuda tensor")
    _check(load().waveal_prefix_attn(cache.desc, batch, q.data_ptr(), _PAIR.pack(q_st[0], q_st[1]), cache.k.data_ptr(), cache.v.data_ptr(),
                                     o.data_ptr(), _PAIR.pack(o_st[0], o_st[1]), _ptr(lse), seq_start.data_ptr(), kv_len.data_ptr(),
                                     _ptr(page_table), prefix_ptr, scale, workspace.data_ptr(), workspace.numel(), _status(dev_status),
                                     _stream(stream)))
    return (o, lse) if return_lse else o


# ------------------------------------------------------------------ whole prompts, pages of the cache

PROMPT_CAUSAL = 1
PROMPT_SELFTEST_LOST_TILE = 256

# waveal_prompt_desc, waveal_fork_desc, waveal_compact_desc as the C compiler lays them out
_PROMPT = struct.Struct("7i4x8q")
_FORK = struct.Struct("4i2q")
_COMPACT = struct.Struct("3i4x2q")


def _here(*tensors):
    """The library works on the current device: tensors of another one are refused."""
    dev = _torch._C._cuda_getDevice()
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise ValueError(f"a tensor is on {t.device}, the current device is cuda:{dev}")


_bytes = {}


def _workspace_bytes(query, *descs):
    """What a size query answers for these descriptors, which alone decide it; the last ones asked for are kept."""
    n = _bytes.get(descs)
    if n is None:
        n = query(*descs)
        if len(_bytes) >= 256:
            _bytes.clear()
        _bytes[descs] = n
    return n


def _new_like(like, stream, *shape):
    """A new tensor of the type of `like`.  Every result has one of its own: who keeps or saves it keeps no other, and no workspace.  (Sizes as arguments, no
    type: 0.9 us each; a shape and a type 1.6, a view of a common block 1.4.)"""
    return like.new_empty(*shape) if stream is None else _new(stream, lambda: like.new_empty(*shape))


def _ints(name, t, shape):
    """address of a contiguous int32 cuda tensor of this shape"""
    if t.dtype is not _torch.int32 or not t.is_cuda:
        raise TypeError(f"{name} must be an int32 cuda tensor")
    if t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous {list(shape)}, got {list(t.shape)}")
    return t.data_ptr()


def _table(name, t):
    """(rows, pages, entries from one row to the next) of a page table"""
    if t.dtype is not _torch.int32 or not t.is_cuda:
        raise TypeError(f"{name} must be an int32 cuda tensor")
    shape, st = t.shape, t.stride()
    if len(st) != 2 or st[1] != 1 and shape[1] > 1:
        raise ValueError(f"{name} must be [rows, pages], a row's pages contiguous")
    return shape[0], shape[1], st[0] if shape[0] > 1 else max(st[0], shape[1])


def _check_workspace(workspace):
    if workspace.dtype is not _torch.uint8 or not workspace.is_cuda or not workspace.is_contiguous():
        raise TypeError("workspace must be a contiguous uint8 cuda tensor")


def prompt_desc(q, k, v, o, batch: int, causal: bool = True, flags: int = 0) -> bytes:
    """The waveal_prompt_desc of a call, from its tensors."""
    _load_torch()
    q_st, k_st, v_st, o_st = _rows("q", q), _rows("k", k), _rows("v", v), _rows("o", o)
    heads, tokens, dim = q.shape
    if k.shape != v.shape or k.shape[1] != tokens or k.shape[2] != dim:
        raise ValueError("k and v must be [kv_heads, tokens, head_dim] with q's tokens and head_dim")
    if k.dtype is not q.dtype or v.dtype is not q.dtype:
        raise TypeError("q, k and v must have one type")
    return _PROMPT.pack(batch, tokens, heads, k.shape[0], dim, _dtype(q), (PROMPT_CAUSAL if causal else 0) | flags, q_st[0], q_st[1], k_st[0], k_st[1],
                        v_st[0], v_st[1], o_st[0], o_st[1])


def prompt_attn_workspace_bytes(desc: bytes) -> int:
    """Bytes for prompt_attn's workspace; desc: prompt_desc of the call."""
    n = ctypes.c_size_t(0)
    _check(load().waveal_prompt_attn_workspace_bytes(desc, ctypes.byref(n)))
    return n.value


def prompt_attn(q, k, v, seq_start, seq_len=None, o=None, lse=None, return_lse: bool = False, causal: bool = True, scale: float = 0.0,
                workspace=None, dev_status=None, flags: int = 0, stream=None):
    """waveal_prompt_attn.  q: [q_heads, tokens, head_dim], k, v: [kv_heads, tokens, head_dim], bf16 or fp16, the tokens of all sequences one
    after another (any strides: a [tokens, heads, head_dim] tensor is passed as x.transpose(0, 1)); seq_start int32 [batch + 1]; seq_len int32
    [batch], where only a sequence's first tokens exist.  Every token attends to its own sequence, up to itself with causal.  Returns o (laid out
    like q unless given), or (o, lse) with return_lse; tokens of no sequence are not written.  What the call allocates belongs to its stream."""
    torch = _load_torch()
    o = _output("o", o, q, stream)
    if seq_start.dim() != 1 or seq_start.shape[0] < 1:
        raise ValueError("seq_start must be [batch + 1]")
    batch = seq_start.shape[0] - 1
    start = _ints("seq_start", seq_start, (batch + 1,))
    lens = None if seq_len is None else _ints("seq_len", seq_len, (batch,))
    desc = prompt_desc(q, k, v, o, batch, causal, flags)
    heads, tokens = q.shape[0], q.shape[1]
    if lse is not None and (lse.dtype is not torch.float32 or lse.shape != (heads, tokens) or not lse.is_cuda or not lse.is_contiguous()):
        raise ValueError("lse must be a contiguous float32 cuda tensor [q_heads, tokens]")
    new_lse = lse is None and return_lse
    if new_lse:
        lse = _new(stream, lambda: q.new_empty((heads, tokens), dtype=torch.float32))
    if workspace is None:
        size = _workspace_bytes(prompt_attn_workspace_bytes, desc)
        workspace = _new_like(q, stream, size // 2)
    else:
        _check_workspace(workspace)
        size = workspace.numel()
    _here(q, k, v, o, lse, seq_start, seq_len, workspace, dev_status)
    _check(load().waveal_prompt_attn(desc, q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), _ptr(lse), start, lens, scale, workspace.data_ptr(), size,
                                     _status(dev_status), _stream(stream)))
    return (o, lse) if return_lse else o


def cache_fork_workspace_bytes(cache_desc: bytes, fork: bytes) -> int:
    """Bytes for cache_fork's workspace: PagedCache.desc and the packed waveal_fork_desc."""
    n = ctypes.c_size_t(0)
    _check(load().waveal_cache_fork_workspace_bytes(cache_desc, fork, ctypes.byref(n)))
    return n.value


def cache_fork(cache: PagedCache, page_table, held_len, page_refs, keep_len, room_len, parents=None, max_pages: Optional[int] = None,
               table_out=None, refs_out=None, workspace=None, dev_status=None, stream=None):
    """waveal_cache_fork: the next step's page table and counts.  page_table int32 [old rows, pages], held_len int32 [old rows]: row r holds the pages
    of its first held_len[r] tokens; page_refs int32 [n_pages]: how many hold each page.  Row b of the new table (as many as keep_len
    has) keeps the first keep_len[b] tokens of row parents[b] (None: row b; negative: a row without pages) and has room for room_len[b].
    Full pages are shared, a page filled in part is copied unless the row is the only one left that holds it, fresh pages are the free ones with the
    lowest numbers.  max_pages: entries of a new row (as many as before unless given).  Returns (page_table, page_refs): new tensors unless given.
    Where the pool runs out (ERR_NO_PAGES in dev_status) entries are -1; the old table is over then too, as its pages may have been written."""
    _load_torch()
    old_rows, old_pages, old_stride = _table("page_table", page_table)
    if keep_len.dim() != 1:
        raise ValueError("keep_len must be [rows]")
    rows = keep_len.shape[0]
    held, refs = _ints("held_len", held_len, (old_rows,)), _ints("page_refs", page_refs, (cache.n_pages,))
    keep, room = _ints("keep_len", keep_len, (rows,)), _ints("room_len", room_len, (rows,))
    parent = None if parents is None else _ints("parents", parents, (rows,))
    pages, n = old_pages if max_pages is None else max_pages, cache.n_pages
    stride = pages
    if table_out is not None:
        new_rows, pages, stride = _table("table_out", table_out)
        if new_rows != rows or max_pages is not None and pages != max_pages:
            raise ValueError("table_out must be [rows of keep_len, max_pages]")
    desc = _FORK.pack(old_rows, rows, old_pages, pages, old_stride, stride)
    size = _workspace_bytes(cache_fork_workspace_bytes, cache.desc, desc)
    if table_out is None:
        table_out = _new_like(page_refs, stream, rows, pages)
    if refs_out is None:
        refs_out = _new_like(page_refs, stream, n)
        refs_ptr = refs_out.data_ptr()
    else:
        refs_ptr = _ints("refs_out", refs_out, (n,))
    if workspace is None:
        workspace = _new_like(page_refs, stream, size // 4)
    else:
        _check_workspace(workspace)
        size = workspace.numel()
    _here(cache.k, cache.v, page_table, held_len, page_refs, keep_len, room_len, parents, table_out, refs_out, workspace, dev_status)
    _check(load().waveal_cache_fork(cache.desc, desc, cache.k.data_ptr(), cache.v.data_ptr(), page_table.data_ptr(), held, refs, parent, keep, room,
                                    table_out.data_ptr(), refs_ptr, workspace.data_ptr(), size, _status(dev_status), _stream(stream)))
    return table_out, refs_out


class Compacted(NamedTuple):
    page_table: object      # [rows, pages] or None
    prefix_pages: object    # or None
    page_refs: object       # [n_pages]
    place: object           # [n_pages]: every page's new number, -1 for a free one
    used: object            # [1]: pages in use; they are the first ones now


def cache_compact_workspace_bytes(cache_desc: bytes) -> int:
    """Bytes for cache_compact's workspace: PagedCache.desc."""
    n = ctypes.c_size_t(0)
    _check(load().waveal_cache_compact_workspace_bytes(cache_desc, ctypes.byref(n)))
    return n.value


def cache_compact(cache: PagedCache, page_refs, page_table=None, prefix_pages=None, workspace=None, stream=None) -> Compacted:
    """waveal_cache_compact: moves the pages that are in use (page_refs int32 [n_pages] above zero) to the lowest numbers and translates
    page_table int32 [rows, pages] and the list prefix_pages, where given.  Returns new tensors (Compacted); other lists of pages are translated by
    `place`."""
    _load_torch()
    refs = _ints("page_refs", page_refs, (cache.n_pages,))
    n = cache.n_pages
    rows = pages = old_stride = count = 0
    if page_table is not None:
        rows, pages, old_stride = _table("page_table", page_table)
    if prefix_pages is not None:
        count = prefix_pages.numel()
        _ints("prefix_pages", prefix_pages, (count,))
    size = _workspace_bytes(cache_compact_workspace_bytes, cache.desc)
    table = None if page_table is None else _new_like(page_refs, stream, rows, pages)
    prefix = None if prefix_pages is None else _new_like(page_refs, stream, count)
    refs_out, place, used = _new_like(page_refs, stream, n), _new_like(page_refs, stream, n), _new_like(page_refs, stream, 1)
    if workspace is None:
        workspace = _new_like(page_refs, stream, size // 4)
    else:
        _check_workspace(workspace)
        size = workspace.numel()
    _here(cache.k, cache.v, page_refs, page_table, prefix_pages, workspace)
    _check(load().waveal_cache_compact(cache.desc, _COMPACT.pack(rows, pages, count, old_stride, pages), cache.k.data_ptr(), cache.v.data_ptr(), refs,
                                       _ptr(page_table), _ptr(prefix_pages), refs_out.data_ptr(), _ptr(table), _ptr(prefix), place.data_ptr(),
                                       used.data_ptr(), workspace.data_ptr(), size, _stream(stream)))
    return Compacted(table, prefix, refs_out, place, used)


def cache_copy(to: PagedCache, to_pages, source: PagedCache, from_pages, dev_status=None, stream=None):
    """waveal_cache_copy: page from_pages[i] of `source` goes to page to_pages[i] of `to` (which may be the same cache); -1 on either side:
    nothing.  int32 lists; a page that is written stands in to_pages once and, in one cache, not in from_pages."""
    _load_torch()
    if to.dtype is not source.dtype:
        raise TypeError("the caches must have one type")
    count = to_pages.numel()
    t, f = _ints("to_pages", to_pages, (count,)), _ints("from_pages", from_pages, (count,))
    _here(to.k, to.v, source.k, source.v, to_pages, from_pages, dev_status)
    _check(load().waveal_cache_copy(to.desc, source.desc, count, source.k.data_ptr(), source.v.data_ptr(), to.k.data_ptr(), to.v.data_ptr(), f, t,
                                    _status(dev_status), _stream(stream)))
