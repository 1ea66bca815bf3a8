"""ctypes binding over libsalicache.so: argument marshalling only.

Every function below has the name of the C entry point it calls and passes device pointers of
torch tensors plus the current CUDA stream.  Nothing is computed in Python and there is no CPU
fallback: a missing or unloadable library raises at import of this module's `lib()`.
"""
from __future__ import annotations

import ctypes as C
import os

from . import build as _build

REUSE, PRUNE, INT4, INT8, FP16 = 0, 1, 2, 3, 4

F16, BF16 = 0, 1
HALVES, NEIGHBOURS = 0, 1

E_NULL, E_SHAPE, E_ALIGN, E_PARAM, E_CUDA, E_CAPACITY, E_NOCONVERGE, E_NOMEM, E_EVICTED = -1, -2, -3, -4, -5, -6, -7, -8, -9


class SalicacheError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {lib().salicache_strerror(status).decode()} ({status})")


class Params(C.Structure):
    _fields_ = [
        ("H", C.c_int32), ("W", C.c_int32), ("patch", C.c_int32), ("n_images", C.c_int32),
        ("max_batch", C.c_int32), ("chunk_frames", C.c_int32),
        ("pyr_levels", C.c_int32), ("poly_n", C.c_int32), ("poly_sigma", C.c_double),
        ("win", C.c_int32), ("iters", C.c_int32), ("eps_det", C.c_double),
        ("canny_lo", C.c_int32), ("canny_hi", C.c_int32), ("var_radius", C.c_int32),
        ("sigma_ref", C.c_double), ("w_edge", C.c_double), ("w_color", C.c_double),
        ("hyst_max_iters", C.c_int32),
        ("tau_t", C.c_float), ("theta_R", C.c_float), ("tau_high", C.c_float), ("tau_med", C.c_float),
        ("tau_low", C.c_float), ("patch_reuse", C.c_int32),
        ("L", C.c_int32), ("heads", C.c_int32), ("head_dim", C.c_int32), ("group", C.c_int32),
        ("color_norm", C.c_int32), ("color_kappa", C.c_double), ("color_sigma_min", C.c_double),
    ]


class Pools(C.Structure):
    _fields_ = [
        ("fp16_pool", C.c_void_p), ("int8_codes", C.c_void_p), ("int8_scale", C.c_void_p),
        ("int4_codes", C.c_void_p), ("int4_sz", C.c_void_p),
        ("cap_fp16", C.c_int64), ("cap_int8", C.c_int64), ("cap_int4", C.c_int64), ("ring", C.c_int32),
        ("d_fill", C.c_void_p),
    ]


class Pages(C.Structure):
    device = None        # CUDA device of the pages, where known
    _fields_ = [
        ("d_data", C.c_void_p), ("d_scale", C.c_void_p),
        ("n_pages", C.c_int32), ("page", C.c_int32), ("heads", C.c_int32), ("head_dim", C.c_int32),
        ("format", C.c_int32), ("dtype", C.c_int32),
    ]


class SeqsC(C.Structure):
    device = None
    _fields_ = [
        ("n_seqs", C.c_int32), ("table_width", C.c_int32), ("n_rows", C.c_int32),
        ("d_row_start", C.c_void_p), ("d_len", C.c_void_p), ("d_table", C.c_void_p),
    ]


class Rotary(C.Structure):
    """Radians per position of every pair, the axis of the position that turns it (none: all on the one there is), and how the
    pairs lie (HALVES or NEIGHBOURS)."""
    _fields_ = [
        ("freq", C.c_double * 64), ("axis", C.c_uint8 * 64), ("pairs", C.c_int32), ("n_axes", C.c_int32), ("pairing", C.c_int32),
    ]

    def __init__(self, freq, axis=None, n_axes: int = 1, pairing: int = HALVES):
        freq = [float(x) for x in freq]
        axis = [0] * len(freq) if axis is None else [int(x) for x in axis]
        if len(freq) > 64 or len(axis) != len(freq) or any(not 0 <= x < 256 for x in axis):
            raise ValueError("at most 64 frequencies, and an axis for each, expected")
        super().__init__((C.c_double * 64)(*freq), (C.c_uint8 * 64)(*axis), len(freq), n_axes, pairing)


EXPORTS = [
    "salicache_default_params", "salicache_create", "salicache_destroy", "salicache_strerror",
    "salicache_tokens_per_frame", "salicache_launch_count", "salicache_flow_score", "salicache_saliency", "salicache_select",
    "salicache_pack_kv", "salicache_unpack_kv", "salicache_poll_status", "salicache_saliency_noalloc",
    "salicache_frame_redundancy", "salicache_source_frames", "salicache_diff_score", "salicache_attend",
    "salicache_select_anchored", "salicache_select_ranked", "salicache_attend_gqa", "salicache_select_anchored_batch",
    "salicache_frames_resident", "salicache_tokens_live", "salicache_paged_write", "salicache_paged_read",
    "salicache_paged_attend", "salicache_paged_work_bytes", "salicache_paged_wait_limit", "salicache_paged_write_rotary",
    "salicache_paged_attend_tree", "salicache_paged_weigh", "salicache_select_heavy", "salicache_paged_keep",
]

_lib = None


def lib():
    """Loads (building first if the sources are newer) the CUDA library.  Fails loudly if it cannot."""
    global _lib
    if _lib is None:
        path = _build.LIB
        if os.path.exists(os.path.join(_build.CSRC, "api.cu")) and _build.nvcc_path() is not None:
            path = _build.build()
        if not os.path.exists(path):
            raise ImportError(f"{path} is missing: build it with `python -m paper_2602_14236_b200.build`; "
                              "there is no CPU fallback")
        _lib = C.CDLL(path)
        _lib.salicache_strerror.restype = C.c_char_p
        _lib.salicache_strerror.argtypes = [C.c_int]
        _lib.salicache_create.argtypes = [C.POINTER(C.c_void_p), C.POINTER(Params)]
        _lib.salicache_destroy.argtypes = [C.c_void_p]
        _lib.salicache_tokens_per_frame.argtypes = [C.c_void_p]
        _lib.salicache_default_params.argtypes = [C.POINTER(Params)]
        _lib.salicache_launch_count.argtypes = [C.c_void_p]
        _lib.salicache_launch_count.restype = C.c_int64
        vp, i32, i64 = C.c_void_p, C.c_int, C.c_int64
        _lib.salicache_flow_score.argtypes = [vp, vp, vp, i32, vp, vp, vp]
        _lib.salicache_saliency.argtypes = [vp, vp, i32, vp, vp, vp]
        _lib.salicache_diff_score.argtypes = [vp, vp, vp, i32, vp, vp]
        _lib.salicache_frame_redundancy.argtypes = [vp, vp, i32, i32, vp, vp]
        _lib.salicache_source_frames.argtypes = [vp, vp, i32, i32, vp, vp, vp]
        _lib.salicache_select.argtypes = [vp, vp, vp, i32, i32, vp, vp, vp, vp, vp, vp, vp]
        _lib.salicache_select_ranked.argtypes = [vp, vp, vp, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp]
        _lib.salicache_select_anchored_batch.argtypes = [vp, vp, vp, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp]
        _lib.salicache_select_anchored.argtypes = [vp, vp, vp, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp]
        _lib.salicache_pack_kv.argtypes = [vp, vp, vp, i64, vp, vp, vp, i32, C.POINTER(Pools), vp]
        _lib.salicache_unpack_kv.argtypes = [vp, C.POINTER(Pools), vp, vp, vp, vp, i32, i32, vp, vp, i64, vp]
        _lib.salicache_poll_status.argtypes = [vp, vp]
        _lib.salicache_attend.argtypes = [vp, vp, C.POINTER(Pools), vp, vp, vp]
        _lib.salicache_attend_gqa.argtypes = [vp, vp, i32, C.POINTER(Pools), vp, vp, vp]
        _lib.salicache_saliency_noalloc.argtypes = [C.POINTER(Params), vp, i32, vp, vp, vp]
        _lib.salicache_frames_resident.argtypes = [vp, vp, vp, i32, C.POINTER(Pools), vp, vp]
        _lib.salicache_paged_write.argtypes = [vp, C.POINTER(Pages), C.POINTER(SeqsC), vp, vp, i64, i64, vp]
        _lib.salicache_paged_read.argtypes = [vp, C.POINTER(Pages), C.POINTER(SeqsC), vp, vp, i64, i64, vp]
        _lib.salicache_paged_attend.argtypes = [vp, C.POINTER(Pages), C.POINTER(SeqsC), vp, i64, i32, C.c_float, i32, i32, vp, i64,
                                                vp, vp, i64, vp]
        _lib.salicache_paged_write_rotary.argtypes = [vp, C.POINTER(Pages), C.POINTER(SeqsC), C.POINTER(Rotary), vp, vp, i64, i32, vp,
                                                      i64, vp, vp, i64, i64, vp]
        _lib.salicache_paged_attend_tree.argtypes = [vp, C.POINTER(Pages), C.POINTER(SeqsC), vp, i32, vp, i64, i32, C.c_float, i32, i32,
                                                     vp, i64, vp, vp, i64, vp]
        _lib.salicache_paged_weigh.argtypes = [vp, C.POINTER(Pages), C.POINTER(SeqsC), vp, i64, i32, C.c_float, vp, C.c_float, vp, vp,
                                               i64, vp, i64, vp]
        _lib.salicache_select_heavy.argtypes = [vp, vp, i64, i32, i32, vp, i32, i32, i32, vp, vp, vp]
        _lib.salicache_paged_keep.argtypes = [vp, C.POINTER(Pages), C.POINTER(SeqsC), vp, i32, i32, vp, vp, C.POINTER(SeqsC), vp, vp,
                                              i64, vp]
        _lib.salicache_paged_wait_limit.argtypes = [vp, i32]
        _lib.salicache_paged_work_bytes.argtypes = [vp, C.POINTER(Pages), i32]
        _lib.salicache_paged_work_bytes.restype = i64
        _lib.salicache_tokens_live.argtypes = [vp, vp, i32, i32, vp, i32, vp, vp]
    return _lib


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _here():
    """The current device and its current stream, the way the paged calls ask for them: once per call."""
    global _torch_c
    if _torch_c is None:
        import torch
        torch.cuda.current_stream()
        _torch_c = torch._C
    dev = _torch_c._cuda_getDevice()
    return dev, _torch_c._cuda_getCurrentRawStream(dev)


_torch_c = None


def _dptr(t, dev, dtype, n):
    """The address of `n` elements of type `dtype` (None: bytes, of any type) from a tensor's first on, on device `dev`.  The C
    entry points see an address only: not whose memory it is, what it holds or where it ends."""
    if t is None:
        return None
    if t.get_device() != dev:
        raise ValueError(f"a tensor on cuda:{dev}, the current device, expected, got one on {t.device}")
    if dtype is None:
        n = -(-n // t.element_size())
    elif t.dtype is not dtype:
        raise ValueError(f"a tensor of type {dtype} expected, got {t.dtype}")
    # a tensor without gaps, or a part of a wider one: rows may go on behind the view's end, not behind its memory's
    if t.numel() < n or not t.is_contiguous():
        held = t.untyped_storage().nbytes() // t.element_size() - t.storage_offset()
        if held < n:
            raise ValueError(f"memory for {n} elements expected from the tensor's first on, got {held}")
    return t.data_ptr()


def _types():
    global _torch_types
    import torch
    _torch_types = {F16: torch.float16, BF16: torch.bfloat16, "lse": torch.float32, "i32": torch.int32, "i64": torch.int64}
    return _torch_types


_torch_types = None


def _batch(pages: Pages, seqs: SeqsC, dev: int, stream):
    """Refuses pages, offsets or a stream of another device than the current one (structs filled by hand name none)."""
    for what, at in (("pages", pages.device), ("offsets", seqs.device), ("stream", None if stream is None else stream.device_index)):
        if at is not None and at != dev:
            raise ValueError(f"{what} of cuda:{dev}, the current device, expected, got cuda:{at}")


def _stream(stream=None):
    import torch
    s = torch.cuda.current_stream() if stream is None else stream
    return C.c_void_p(s.cuda_stream)


def _check(status: int, where: str):
    if status != 0:
        raise SalicacheError(status, where)


def salicache_default_params(**overrides) -> Params:
    p = Params()
    _check(lib().salicache_default_params(C.byref(p)), "salicache_default_params")
    for k, v in overrides.items():
        if not hasattr(p, k):
            raise AttributeError(k)
        setattr(p, k, v)
    return p


class Context:
    """Owns a salicache_ctx (scratch only).  Create it with the wanted device current."""

    def __init__(self, params: Params):
        self.params = params
        self._h = C.c_void_p()
        _check(lib().salicache_create(C.byref(self._h), C.byref(params)), "salicache_create")
        self.n_tok = int(lib().salicache_tokens_per_frame(self._h))
        self.HD = params.heads * params.head_dim

    def close(self):
        if self._h:
            lib().salicache_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def launch_count(self) -> int:
        return int(lib().salicache_launch_count(self._h))

    @property
    def handle(self):
        return self._h


def salicache_flow_score(ctx: Context, d_prev, d_cur, B: int, d_deltaP, d_flow=None, stream=None):
    _check(lib().salicache_flow_score(ctx.handle, _ptr(d_prev), _ptr(d_cur), B, _ptr(d_deltaP), _ptr(d_flow),
                                      _stream(stream)), "salicache_flow_score")


def salicache_diff_score(ctx: Context, d_prev, d_cur, B: int, d_deltaP, stream=None):
    _check(lib().salicache_diff_score(ctx.handle, _ptr(d_prev), _ptr(d_cur), B, _ptr(d_deltaP), _stream(stream)),
           "salicache_diff_score")


def salicache_saliency(ctx: Context, d_frames, B: int, d_s, d_skip=None, stream=None):
    _check(lib().salicache_saliency(ctx.handle, _ptr(d_frames), B, _ptr(d_s), _ptr(d_skip), _stream(stream)),
           "salicache_saliency")


def salicache_frame_redundancy(ctx: Context, d_deltaP, B: int, first_has_no_prev: bool, d_frame_redundant, stream=None):
    _check(lib().salicache_frame_redundancy(ctx.handle, _ptr(d_deltaP), B, int(first_has_no_prev),
                                            _ptr(d_frame_redundant), _stream(stream)), "salicache_frame_redundancy")


def salicache_saliency_noalloc(params: Params, d_frames, B: int, d_s, d_status=None, stream=None):
    """Spatial score for hosts that cannot allocate device memory (no context needed): at most
    NOALLOC_MAX_FRAMES frames of at most NOALLOC_MAX_SIDE pixels a side per call.  Calls on one
    device share a fixed scratch array inside the library, so they must not overlap on the GPU."""
    _check(lib().salicache_saliency_noalloc(C.byref(params), _ptr(d_frames), B, _ptr(d_s), _ptr(d_status),
                                            _stream(stream)), "salicache_saliency_noalloc")


NOALLOC_MAX_FRAMES, NOALLOC_MAX_SIDE = 8, 336


def salicache_source_frames(ctx: Context, d_decision, B: int, first_frame: int, d_carry, d_src, stream=None):
    _check(lib().salicache_source_frames(ctx.handle, _ptr(d_decision), B, first_frame, _ptr(d_carry), _ptr(d_src),
                                         _stream(stream)), "salicache_source_frames")


def salicache_select(ctx: Context, d_deltaP, d_s, B: int, first_has_no_prev: bool, d_decision, d_idx, d_counts,
                     d_frame_redundant, d_row_offset, d_fill, stream=None):
    _check(lib().salicache_select(ctx.handle, _ptr(d_deltaP), _ptr(d_s), B, int(first_has_no_prev), _ptr(d_decision),
                                  _ptr(d_idx), _ptr(d_counts), _ptr(d_frame_redundant), _ptr(d_row_offset),
                                  _ptr(d_fill), _stream(stream)), "salicache_select")


def salicache_select_ranked(ctx: Context, d_deltaP, d_s, B: int, first_has_no_prev: bool, shares_permille, d_decision, d_idx,
                            d_counts, d_frame_redundant, d_row_offset, d_fill, stream=None):
    pm16, pm8, pm4 = (int(x) for x in shares_permille)
    _check(lib().salicache_select_ranked(ctx.handle, _ptr(d_deltaP), _ptr(d_s), B, int(first_has_no_prev), pm16, pm8, pm4,
                                         _ptr(d_decision), _ptr(d_idx), _ptr(d_counts), _ptr(d_frame_redundant),
                                         _ptr(d_row_offset), _ptr(d_fill), _stream(stream)), "salicache_select_ranked")


def salicache_select_anchored(ctx: Context, d_frames, d_s, B: int, first_has_no_prev: bool, d_anchor, d_deltaP, d_decision,
                              d_idx, d_counts, d_frame_redundant, d_row_offset, d_fill, stream=None):
    _check(lib().salicache_select_anchored(ctx.handle, _ptr(d_frames), _ptr(d_s), B, int(first_has_no_prev), _ptr(d_anchor),
                                           _ptr(d_deltaP), _ptr(d_decision), _ptr(d_idx), _ptr(d_counts),
                                           _ptr(d_frame_redundant), _ptr(d_row_offset), _ptr(d_fill), _stream(stream)),
           "salicache_select_anchored")


def salicache_select_anchored_batch(ctx: Context, d_frames, d_s, n_videos: int, B: int, first_has_no_prev: bool, d_anchor, d_deltaP,
                                    d_decision, d_idx, d_counts, d_frame_redundant, d_row_offset, d_fill, stream=None):
    _check(lib().salicache_select_anchored_batch(ctx.handle, _ptr(d_frames), _ptr(d_s), n_videos, B, int(first_has_no_prev),
                                                 _ptr(d_anchor), _ptr(d_deltaP), _ptr(d_decision), _ptr(d_idx), _ptr(d_counts),
                                                 _ptr(d_frame_redundant), _ptr(d_row_offset), _ptr(d_fill), _stream(stream)),
           "salicache_select_anchored_batch")


def salicache_pack_kv(ctx: Context, d_K, d_V, frame_stride: int, d_idx, d_counts, d_row_offset, B: int, pools: Pools,
                      stream=None):
    _check(lib().salicache_pack_kv(ctx.handle, _ptr(d_K), _ptr(d_V), frame_stride, _ptr(d_idx), _ptr(d_counts),
                                   _ptr(d_row_offset), B, C.byref(pools), _stream(stream)), "salicache_pack_kv")


def salicache_unpack_kv(ctx: Context, pools: Pools, d_idx, d_counts, d_decision, d_row_offset, B: int,
                        zero_fill_pruned: bool, d_K_out, d_V_out, frame_stride: int, stream=None):
    _check(lib().salicache_unpack_kv(ctx.handle, C.byref(pools), _ptr(d_idx), _ptr(d_counts), _ptr(d_decision),
                                     _ptr(d_row_offset), B, int(zero_fill_pruned), _ptr(d_K_out), _ptr(d_V_out),
                                     frame_stride, _stream(stream)), "salicache_unpack_kv")


def salicache_attend(ctx: Context, d_q, pools: Pools, d_fill, d_out, stream=None):
    _check(lib().salicache_attend(ctx.handle, _ptr(d_q), C.byref(pools), _ptr(d_fill), _ptr(d_out), _stream(stream)),
           "salicache_attend")


def salicache_attend_gqa(ctx: Context, d_q, q_per_kv: int, pools: Pools, d_fill, d_out, stream=None):
    _check(lib().salicache_attend_gqa(ctx.handle, _ptr(d_q), int(q_per_kv), C.byref(pools), _ptr(d_fill), _ptr(d_out),
                                      _stream(stream)), "salicache_attend_gqa")


def salicache_frames_resident(ctx: Context, d_counts, d_row_offset, B: int, pools: Pools, d_resident, stream=None):
    _check(lib().salicache_frames_resident(ctx.handle, _ptr(d_counts), _ptr(d_row_offset), B, C.byref(pools), _ptr(d_resident),
                                           _stream(stream)), "salicache_frames_resident")


def salicache_tokens_live(ctx: Context, d_src, B: int, first_frame: int, d_resident_table, n_table: int, d_live, stream=None):
    _check(lib().salicache_tokens_live(ctx.handle, _ptr(d_src), B, first_frame, _ptr(d_resident_table), n_table, _ptr(d_live),
                                       _stream(stream)), "salicache_tokens_live")


def _paged_move(name: str, ctx: Context, pages: Pages, seqs: SeqsC, d_K, d_V, k_stride: int, v_stride: int, stream):
    dev, st = _here()
    if not pages.device == seqs.device == dev or stream is not None:
        _batch(pages, seqs, dev, stream)
    t, gaps, width = (_torch_types or _types()).get(pages.dtype), seqs.n_rows - 1, pages.heads * pages.head_dim
    rc = getattr(_lib or lib(), name)(ctx.handle, pages, seqs, _dptr(d_K, dev, t, gaps * k_stride + width if gaps >= 0 else 0),
                                      _dptr(d_V, dev, t, gaps * v_stride + width if gaps >= 0 else 0), k_stride, v_stride,
                                      st if stream is None else stream.cuda_stream)
    if rc:
        raise SalicacheError(rc, name)


def salicache_paged_write(ctx: Context, pages: Pages, seqs: SeqsC, d_K, d_V, k_stride: int, v_stride: int, stream=None):
    _paged_move("salicache_paged_write", ctx, pages, seqs, d_K, d_V, k_stride, v_stride, stream)


def salicache_paged_read(ctx: Context, pages: Pages, seqs: SeqsC, d_K_out, d_V_out, k_stride: int, v_stride: int, stream=None):
    _paged_move("salicache_paged_read", ctx, pages, seqs, d_K_out, d_V_out, k_stride, v_stride, stream)


def _span(rows: int, stride: int, width: int) -> int:
    """Elements from the first of `rows` rows to the end of the last one."""
    return (rows - 1) * stride + width if rows > 0 else 0


def salicache_paged_write_rotary(ctx: Context, pages: Pages, seqs: SeqsC, rotary: Rotary, d_pos, d_q, q_stride: int, q_per_kv: int,
                                 d_q_out, q_out_stride: int, d_K, d_V, k_stride: int, v_stride: int, stream=None):
    """d_q None: no rows of q."""
    dev, st = _here()
    if not pages.device == seqs.device == dev or stream is not None:
        _batch(pages, seqs, dev, stream)
    types, rows, width = _torch_types or _types(), seqs.n_rows, pages.heads * pages.head_dim
    t = types.get(pages.dtype)
    q, q_out = (None, None) if d_q is None else (_dptr(d_q, dev, t, _span(rows, q_stride, width * q_per_kv)),
                                                 _dptr(d_q_out, dev, t, _span(rows, q_out_stride, width * q_per_kv)))
    rc = (_lib or lib()).salicache_paged_write_rotary(
        ctx.handle, pages, seqs, rotary, _dptr(d_pos, dev, types["i32"], rows * rotary.n_axes), q, q_stride, q_per_kv, q_out, q_out_stride,
        _dptr(d_K, dev, t, _span(rows, k_stride, width)), _dptr(d_V, dev, t, _span(rows, v_stride, width)), k_stride, v_stride,
        st if stream is None else stream.cuda_stream)
    if rc:
        raise SalicacheError(rc, "salicache_paged_write_rotary")


def salicache_paged_work_bytes(ctx: Context, pages: Pages, q_per_kv: int) -> int:
    n = int(lib().salicache_paged_work_bytes(ctx.handle, C.byref(pages), q_per_kv))
    if n < 0:
        raise SalicacheError(n, "salicache_paged_work_bytes")
    return n


def salicache_paged_attend(ctx: Context, pages: Pages, seqs: SeqsC, d_q, q_stride: int, q_per_kv: int, softmax_scale: float,
                           window: int, sinks: int, d_out, out_stride: int, d_lse, d_work, work_bytes: int, stream=None):
    dev, st = _here()
    if not pages.device == seqs.device == dev or stream is not None:
        _batch(pages, seqs, dev, stream)
    types, rows, heads = _torch_types or _types(), seqs.n_rows, pages.heads * q_per_kv
    t, gaps, width = types.get(pages.dtype), rows - 1, heads * pages.head_dim
    rc = (_lib or lib()).salicache_paged_attend(
        ctx.handle, pages, seqs, _dptr(d_q, dev, t, gaps * q_stride + width if rows > 0 else 0), q_stride, q_per_kv, softmax_scale,
        window, sinks, _dptr(d_out, dev, t, gaps * out_stride + width if rows > 0 else 0), out_stride,
        _dptr(d_lse, dev, types["lse"], rows * heads), _dptr(d_work, dev, None, work_bytes), work_bytes,
        st if stream is None else stream.cuda_stream)
    if rc:
        raise SalicacheError(rc, "salicache_paged_attend")


def salicache_paged_attend_tree(ctx: Context, pages: Pages, seqs: SeqsC, d_tree, tree_words: int, d_q, q_stride: int, q_per_kv: int,
                                softmax_scale: float, window: int, sinks: int, d_out, out_stride: int, d_lse, d_work, work_bytes: int,
                                stream=None):
    """d_tree: int64, whose bits are taken as they are."""
    dev, st = _here()
    if not pages.device == seqs.device == dev or stream is not None:
        _batch(pages, seqs, dev, stream)
    types, rows, heads = _torch_types or _types(), seqs.n_rows, pages.heads * q_per_kv
    t, width = types.get(pages.dtype), heads * pages.head_dim
    rc = (_lib or lib()).salicache_paged_attend_tree(
        ctx.handle, pages, seqs, _dptr(d_tree, dev, types["i64"], rows * tree_words), tree_words,
        _dptr(d_q, dev, t, _span(rows, q_stride, width)), q_stride, q_per_kv, softmax_scale, window, sinks,
        _dptr(d_out, dev, t, _span(rows, out_stride, width)), out_stride, _dptr(d_lse, dev, types["lse"], rows * heads),
        _dptr(d_work, dev, None, work_bytes), work_bytes, st if stream is None else stream.cuda_stream)
    if rc:
        raise SalicacheError(rc, "salicache_paged_attend_tree")


def salicache_paged_weigh(ctx: Context, pages: Pages, seqs: SeqsC, d_q, q_stride: int, q_per_kv: int, softmax_scale: float, d_lse,
                          decay: float, d_weight_in, d_weight_out, weight_stride: int, d_work, work_bytes: int, stream=None):
    """d_weight_in None: zeros."""
    dev, st = _here()
    if not pages.device == seqs.device == dev or stream is not None:
        _batch(pages, seqs, dev, stream)
    types, rows, heads = _torch_types or _types(), seqs.n_rows, pages.heads * q_per_kv
    f32, held = types["lse"], seqs.n_seqs * pages.heads * weight_stride
    rc = (_lib or lib()).salicache_paged_weigh(
        ctx.handle, pages, seqs, _dptr(d_q, dev, types.get(pages.dtype), _span(rows, q_stride, heads * pages.head_dim)), q_stride, q_per_kv,
        softmax_scale, _dptr(d_lse, dev, f32, rows * heads), decay, _dptr(d_weight_in, dev, f32, held), _dptr(d_weight_out, dev, f32, held),
        weight_stride, _dptr(d_work, dev, None, work_bytes), work_bytes, st if stream is None else stream.cuda_stream)
    if rc:
        raise SalicacheError(rc, "salicache_paged_weigh")


def salicache_select_heavy(ctx: Context, d_weight, weight_stride: int, heads: int, n_seqs: int, d_len, budget: int, sinks: int,
                           recent: int, d_keep, d_kept, stream=None):
    dev, st = _here()
    if stream is not None:
        _batch(Pages(), SeqsC(), dev, stream)
    types = _torch_types or _types()
    i32 = types["i32"]
    rc = (_lib or lib()).salicache_select_heavy(
        ctx.handle, _dptr(d_weight, dev, types["lse"], n_seqs * heads * weight_stride), weight_stride, heads, n_seqs,
        _dptr(d_len, dev, i32, n_seqs), budget, sinks, recent, _dptr(d_keep, dev, i32, n_seqs * heads * budget),
        _dptr(d_kept, dev, i32, n_seqs), st if stream is None else stream.cuda_stream)
    if rc:
        raise SalicacheError(rc, "salicache_select_heavy")


def salicache_paged_keep(ctx: Context, pages: Pages, seqs: SeqsC, d_keep, keep_heads: int, keep_width: int, d_first, d_kept, to,
                         d_weight_in=None, d_weight_out=None, weight_stride: int = 0, stream=None):
    """to: the SeqsC of the pages they go into, or None: in place.  d_first None: from position 0 on."""
    dev, st = _here()
    if not pages.device == seqs.device == dev or stream is not None:
        _batch(pages, seqs, dev, stream)
    if to is not None and to.device != dev:
        _batch(pages, to, dev, stream)
    types, n = _torch_types or _types(), seqs.n_seqs
    i32, f32, held = types["i32"], types["lse"], n * pages.heads * weight_stride
    rc = (_lib or lib()).salicache_paged_keep(
        ctx.handle, pages, seqs, _dptr(d_keep, dev, i32, n * keep_heads * keep_width), keep_heads, keep_width, _dptr(d_first, dev, i32, n),
        _dptr(d_kept, dev, i32, n), to, _dptr(d_weight_in, dev, f32, held), _dptr(d_weight_out, dev, f32, held), weight_stride,
        st if stream is None else stream.cuda_stream)
    if rc:
        raise SalicacheError(rc, "salicache_paged_keep")


def salicache_paged_wait_limit(ctx: Context, tries: int):
    _check(lib().salicache_paged_wait_limit(ctx.handle, tries), "salicache_paged_wait_limit")


def salicache_poll_status(ctx: Context, stream=None) -> int:
    return int(lib().salicache_poll_status(ctx.handle, _stream(stream)))


class PoolSet:
    """Device pools as torch tensors (memory only) plus the C struct that points at them."""

    def __init__(self, L: int, HD: int, cap16: int, cap8: int, cap4: int, ring: bool = False, device="cuda", G: int = 128,
                 fill=None):
        import torch
        ng = HD // G
        self.L, self.HD, self.G = L, HD, G
        self.cap = (cap16, cap8, cap4)
        z = lambda shape, dt: torch.zeros(shape, dtype=dt, device=device)
        self.fp16_pool = z((L, 2, max(cap16, 1), HD), torch.float16)
        self.int8_codes = z((L, 2, max(cap8, 1), HD), torch.int8)
        self.int8_scale = z((L, 2, max(cap8, 1), ng), torch.float16)
        self.int4_codes = z((L, 2, max(cap4, 1), HD // 2), torch.uint8)
        self.int4_sz = z((L, 2, max(cap4, 1), ng, 2), torch.float16)
        self.c = Pools(self.fp16_pool.data_ptr(), self.int8_codes.data_ptr(), self.int8_scale.data_ptr(),
                       self.int4_codes.data_ptr(), self.int4_sz.data_ptr(), cap16, cap8, cap4, int(ring),
                       None if fill is None else fill.data_ptr())
        self.fill = fill              # keeps the tensor alive

    def nbytes(self) -> int:
        return sum(t.numel() * t.element_size() for t in
                   (self.fp16_pool, self.int8_codes, self.int8_scale, self.int4_codes, self.int4_sz))


class PageSet:
    """One layer's pages as torch tensors (memory only) plus the C struct that points at them.  `dtype` is torch.float16
    or torch.bfloat16; existing tensors of the documented shapes can be given as `data` and `scale`."""

    def __init__(self, n_pages: int, page: int, heads: int, head_dim: int, format: int, dtype, device="cuda", data=None, scale=None):
        import torch
        el = {FP16: dtype, INT8: torch.int8, INT4: torch.uint8}[format]
        shape = (n_pages, 2, heads, page, head_dim // 2 if format == INT4 else head_dim)
        sshape = {FP16: None, INT8: shape[:4], INT4: shape[:4] + (2,)}[format]
        self.data = torch.zeros(shape, dtype=el, device=device) if data is None else data
        self.scale = (None if sshape is None else torch.zeros(sshape, dtype=dtype, device=device)) if scale is None else scale
        for t, want, ty in ((self.data, shape, el), (self.scale, sshape, dtype)):
            if t is not None and (not t.is_cuda or t.device != self.data.device):
                raise ValueError(f"pages on one CUDA device expected, got {t.device}")
            if t is not None and (tuple(t.shape) != want or t.dtype != ty or not t.is_contiguous()):
                raise ValueError(f"pages of shape {want} and type {ty} expected, got {tuple(t.shape)}, {t.dtype}")
        self.dtype = dtype
        self.c = Pages(self.data.data_ptr(), None if self.scale is None else self.scale.data_ptr(), n_pages, page, heads, head_dim,
                       format, {torch.float16: F16, torch.bfloat16: BF16}[dtype])
        self.c.device, self.c.memory = self.data.get_device(), (self.data, self.scale)

    def nbytes(self) -> int:
        return sum(t.numel() * t.element_size() for t in (self.data, self.scale) if t is not None)


class Seqs:
    """A ragged batch: keeps the three int32 device tensors alive beside the C struct that points at them."""

    def __init__(self, row_start, length, table, n_rows: int):
        import torch
        n = table.shape[0]
        for t, want in ((row_start, (n + 1,)), (length, (n,)), (table, tuple(table.shape))):
            if not t.is_cuda or t.device != table.device:
                raise ValueError(f"tensors on one CUDA device expected, got {t.device}")
            if t.dtype != torch.int32 or tuple(t.shape) != want or not t.is_contiguous():
                raise ValueError(f"int32 tensor of shape {want} expected, got {tuple(t.shape)}, {t.dtype}")
        self.row_start, self.length, self.table = row_start, length, table
        self.c = SeqsC(n, table.shape[1], n_rows, row_start.data_ptr(), length.data_ptr(), table.data_ptr())
        self.c.device, self.c.memory = table.get_device(), (row_start, length, table)
