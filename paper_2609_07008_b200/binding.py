"""ctypes binding of librk.so with the same names as the C ABI (argument marshalling only).

Every step of the path runs in the library's CUDA kernels; torch is used for device
memory and streams.  Importing this module fails loudly if the shared library has not been
built (`python paper_2609_07008_b200/build.py`): there is no CPU or eager fallback.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional

import numpy as np
import torch

from . import build as _build

RK_OK = 0
STATUS_NAMES = {0: "RK_OK", 1: "RK_ERR_NULL", 2: "RK_ERR_PROFILE", 3: "RK_ERR_LAYOUT", 4: "RK_ERR_ROWS",
                5: "RK_ERR_ALIGN", 6: "RK_ERR_WORKSPACE", 7: "RK_ERR_UNSUPPORTED", 8: "RK_ERR_CUDA",
                9: "RK_ERR_TIMEOUT"}


class rk_profile(C.Structure):
    _fields_ = [("n_heads", C.c_int32), ("n_groups", C.c_int32), ("group_size", C.c_int32),
                ("d_latent", C.c_int32), ("d_rope", C.c_int32), ("d_v", C.c_int32), ("o_rank", C.c_int32),
                ("d_model", C.c_int32), ("sm_scale", C.c_float), ("rope_base", C.c_float),
                ("global_heads", C.POINTER(C.c_int32))]


class rk_layout(C.Structure):
    _fields_ = [("n_segs", C.c_int32), ("seg_off", C.POINTER(C.c_int64)), ("seg_delta", C.POINTER(C.c_int64)),
                ("seg_has_artifact", C.POINTER(C.c_uint8))]


class rk_policy(C.Structure):
    _fields_ = [("edge_rows", C.c_int32), ("tail_rows", C.c_int64), ("budget_bp", C.c_int32)]


class rk_request_info(C.Structure):
    _fields_ = [("n_rows", C.c_int64), ("n_prot", C.c_int64), ("n_off_rows", C.c_int64),
                ("pairs_global", C.c_int64), ("pairs_local", C.c_int64), ("n_tiles_global", C.c_int32),
                ("n_tiles_local", C.c_int32)]


class rk_layer_buffers(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("kv", "q_g", "q_l", "z_off", "O_g", "O_l", "z_on_g", "z_on_l", "z", "y",
                                          "lse_g", "lse_l", "workspace")] + [("workspace_bytes", C.c_size_t)]


class rk_layer_io(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("req", "kv_host", "q_g_host", "q_l_host", "z_off_host", "W_uv", "W_a", "W_b",
                                          "y_host")]


class rk_cache4_table(C.Structure):
    _fields_ = [("n_segs", C.c_int32), ("n_listed", C.c_int64), ("seg_len", C.c_void_p), ("page_off", C.c_void_p),
                ("page_ids", C.c_void_p)]


class rk_decode_shape(C.Structure):
    _fields_ = [("n_seqs", C.c_int32), ("q_len", C.c_int32), ("n_items", C.c_int32), ("max_tiles", C.c_int32)]


class rk_w4(C.Structure):
    _fields_ = [("n_mat", C.c_int32), ("n_out", C.c_int32), ("k", C.c_int32), ("group", C.c_int32),
                ("codes", C.c_void_p), ("scales", C.c_void_p)]


class rk_route(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_experts", "k", "n_groups", "top_groups", "group_top", "score", "renorm")] + [
        ("scale", C.c_float)]


class rk_q8(C.Structure):
    _fields_ = [("n_mat", C.c_int32), ("n_rows", C.c_int64), ("k", C.c_int32), ("codes", C.c_void_p), ("scales", C.c_void_p)]


CACHE4_PAGE_ROWS = 64
CACHE4_PAGE_BYTES = 26624

EXPORTS = ["rk_version", "rk_status_string", "rk_create", "rk_destroy", "rk_last_error", "rk_poll_status",
           "rk_create_ex", "rk_segmented_merge_phase", "rk_check_selftest", "rk_set_wait_limit_ms", "rk_test_starve_loads", "rk_request_create", "rk_request_destroy", "rk_check_request",
           "rk_request_get_info", "rk_workspace_bytes", "rk_relocate_q", "rk_mla_online_attn",
           "rk_segmented_merge", "rk_group_sliced_proj", "rk_group_sliced_proj_static", "rk_combine_offline",
           "rk_layer_host", "rk_layer_stack_host", "rk_mla_off_workspace_bytes", "rk_mla_off_build",
           "rk_protected_rows_workspace_bytes", "rk_protected_rows", "rk_moe_fanout",
           "rk_cache4_append", "rk_cache4_read", "rk_decode_plan_bytes", "rk_decode_plan",
           "rk_cache4_attn_workspace_bytes", "rk_cache4_attn", "rk_quant4", "rk_matvec4",
           "rk_moe_route", "rk_moe_group", "rk_quant8", "rk_matmul8", "rk_matmul8_experts", "rk_sample"]


def _load() -> C.CDLL:
    # RK_LIBRARY_PATH selects another build of the same library (the bounds-checked one, librk_check.so)
    path = os.environ.get("RK_LIBRARY_PATH") or _build.LIB_PATH
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with `python paper_2609_07008_b200/build.py` "
                           "(there is no fallback path)")
    lib = C.CDLL(path)
    vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
    lib.rk_version.restype = C.c_char_p
    lib.rk_status_string.restype = C.c_char_p
    lib.rk_status_string.argtypes = [C.c_int]
    lib.rk_last_error.restype = C.c_char_p
    lib.rk_last_error.argtypes = [vp]
    lib.rk_create.argtypes = [C.POINTER(rk_profile), C.POINTER(vp)]
    lib.rk_destroy.argtypes = [vp]
    lib.rk_poll_status.argtypes = [vp, vp]
    lib.rk_set_wait_limit_ms.argtypes = [vp, i32]
    lib.rk_test_starve_loads.argtypes = [vp, i32]
    lib.rk_check_selftest.argtypes = [vp, vp]
    lib.rk_create_ex.argtypes = [C.POINTER(rk_profile), C.c_uint32, C.POINTER(vp)]
    lib.rk_segmented_merge_phase.argtypes = [vp, vp, i32, i32, i64, i32, vp, i32, vp, vp, vp, vp, vp]
    lib.rk_request_create.argtypes = [vp, C.POINTER(rk_layout), C.POINTER(i32), i64, C.POINTER(vp)]
    lib.rk_request_destroy.argtypes = [vp]
    lib.rk_check_request.argtypes = [C.POINTER(rk_layout), C.POINTER(i32), i64, C.c_char_p, C.c_size_t]
    lib.rk_request_get_info.argtypes = [vp, C.POINTER(rk_request_info)]
    lib.rk_workspace_bytes.argtypes = [vp, C.POINTER(C.c_size_t)]
    lib.rk_relocate_q.argtypes = [vp, vp, vp, i64, i32, i64, i64, i32, i32, vp, vp]
    lib.rk_mla_online_attn.argtypes = [vp] * 10
    lib.rk_segmented_merge.argtypes = [vp, i32, i64, i32, vp, i32, vp, vp, vp, vp]
    lib.rk_group_sliced_proj.argtypes = [vp] * 9 + [C.c_size_t, vp]
    lib.rk_group_sliced_proj_static.argtypes = [vp] * 9
    lib.rk_combine_offline.argtypes = [vp] * 9
    lib.rk_layer_host.argtypes = [vp] * 9 + [C.POINTER(rk_layer_buffers), vp, vp]
    lib.rk_layer_stack_host.argtypes = [vp, i32, C.POINTER(rk_layer_io), C.POINTER(rk_layer_buffers),
                                        C.POINTER(rk_layer_buffers), vp]
    lib.rk_mla_off_workspace_bytes.argtypes = [vp, i64, C.POINTER(C.c_size_t)]
    lib.rk_mla_off_build.argtypes = [vp, vp, vp, i64, i64, vp, vp, vp, vp, vp, C.c_size_t, vp]
    lib.rk_protected_rows_workspace_bytes.argtypes = [i64, i32, C.POINTER(C.c_size_t)]
    lib.rk_protected_rows.argtypes = [vp, C.POINTER(rk_layout), C.POINTER(rk_policy), vp, i64, vp, vp, vp, vp,
                                      C.c_size_t, vp]
    lib.rk_moe_fanout.argtypes = [vp, vp, i64, C.c_float, i32, vp, vp, vp]
    ptab, pshape, pw4 = C.POINTER(rk_cache4_table), C.POINTER(rk_decode_shape), C.POINTER(rk_w4)
    lib.rk_cache4_append.argtypes = [vp, vp, i64, ptab, vp, i64, vp, i64, vp, i64, vp]
    lib.rk_cache4_read.argtypes = [vp, vp, i64, ptab, vp, i64, vp, vp]
    lib.rk_decode_plan_bytes.argtypes = [vp, pshape, C.POINTER(C.c_size_t)]
    lib.rk_decode_plan.argtypes = [vp, pshape, ptab, i64, vp, vp, vp, vp, vp, C.c_size_t, vp]
    lib.rk_cache4_attn_workspace_bytes.argtypes = [vp, pshape, C.POINTER(C.c_size_t)]
    lib.rk_cache4_attn.argtypes = [vp, pshape, vp, C.c_size_t, vp, i64, vp, vp, vp, vp, C.c_size_t, vp]
    lib.rk_quant4.argtypes = [vp, vp, pw4, vp]
    lib.rk_matvec4.argtypes = [vp, pw4, vp, i64, i64, vp, i64, i32, vp]
    pq8 = C.POINTER(rk_q8)
    lib.rk_moe_route.argtypes = [vp, C.POINTER(rk_route), vp, i32, i64, vp, i64, vp, vp, vp]
    lib.rk_moe_group.argtypes = [vp, vp, vp, i64, i32, i32, vp, vp, vp]
    lib.rk_quant8.argtypes = [vp, vp, i64, pq8, vp]
    lib.rk_matmul8.argtypes = [vp, pq8, pq8, vp, i64, i32, vp]
    lib.rk_matmul8_experts.argtypes = [vp, pq8, pq8, vp, vp, i64, i32, vp, i64, i32, vp]
    lib.rk_sample.argtypes = [vp, vp, i32, i64, i64, i32, vp, vp, vp, vp, vp, vp, vp, vp]
    for name in EXPORTS:
        fn = getattr(lib, name)
        if fn.restype is C.c_int:  # default restype: rk_status
            fn.restype = C.c_int
    return lib


lib = _load()


class RKError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {msg}")
        self.status = status


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    assert t.is_contiguous(), "tensors passed to the library must be contiguous"
    return t.data_ptr()


def _empty(shape, dtype, device):
    """Every buffer the binding allocates on behalf of the caller (outputs, scratch) comes from here, so a
    caller with its own memory pool -- or a test that wants guard zones around the outputs -- can replace it."""
    # strides given: a third less time than torch.empty, which matters for calls of a few microseconds
    if type(shape) is int:
        return _empty_strided((shape,), (1,), dtype=dtype, device=device)
    strides, run = [], 1
    for extent in reversed(shape):
        strides.append(run)
        run *= extent if extent > 1 else 1
    return _empty_strided(shape, strides[::-1], dtype=dtype, device=device)


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


# torch's own short ways to the current device and stream, which a torch without CUDA or a later one may not have
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda device: torch.cuda.current_stream(device).cuda_stream)
_empty_strided = torch.empty_strided


def _quick_stream() -> int:
    """The same stream without building torch's Stream object (for calls that take a few microseconds)."""
    return _raw_stream(_current_device())


def _need(t: torch.Tensor, name: str, dtype, shape, contiguous=True) -> torch.Tensor:
    """Type, shape, layout and device of one argument of a decode call (the C ABI sees pointers only).  shape: None for
    any, else a tuple with -1 for any extent.  Written for speed: a decode step makes a handful of these calls per layer."""
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, not {t.dtype}")
    if shape is not None and (got := t.shape) != shape:
        if len(got) != len(shape):
            raise ValueError(f"{name} must have {len(shape)} dimensions, not {len(got)}")
        for want, have in zip(shape, got):
            if want != -1 and want != have:
                raise ValueError(f"{name} must have the shape {shape} (-1: any), not {tuple(got)}")
    if contiguous and not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if not t.is_cuda or t.get_device() != _current_device():
        raise ValueError(f"{name} must be on the current CUDA device, not on {t.device}")
    return t


def _pages(t: torch.Tensor) -> int:
    """The same checks for the pages of a cache; their number."""
    shape = t.shape
    if t.dtype is not torch.uint8 or len(shape) != 2 or shape[1] != CACHE4_PAGE_BYTES or not t.is_contiguous() or not t.is_cuda or t.get_device() != _current_device():
        _need(t, "pages", torch.uint8, (-1, CACHE4_PAGE_BYTES))
    return shape[0]


def _here(kept, name: str):
    """Tables, plans and weights are kept between calls, and the current device may have changed since they were made."""
    if kept.index != _current_device():
        raise ValueError(f"{name} was made on CUDA device {kept.index}, which is not the current one")


class CacheTable:
    """Segments of a 4-bit paged cache and their pages: device int32 seg_len [S], page_off [S + 1], page_ids [n].
    The tensors are used as they are at the time of each call; their contents may change between calls."""

    def __init__(self, seg_len: torch.Tensor, page_off: torch.Tensor, page_ids: torch.Tensor):
        self.seg_len = _need(seg_len, "seg_len", torch.int32, (-1,))
        self.page_off = _need(page_off, "page_off", torch.int32, (seg_len.numel() + 1,))
        self.page_ids = _need(page_ids, "page_ids", torch.int32, (-1,))
        self.n_segs, self.index = seg_len.numel(), seg_len.get_device()
        self.struct = rk_cache4_table(self.n_segs, page_ids.numel(), _ptr(seg_len), _ptr(page_off), _ptr(page_ids))
        self.ref = C.byref(self.struct)


class DecodePlan:
    """Work list of one decode step (rk_decode_plan): shape, pool size and the device buffer."""

    def __init__(self, shape: rk_decode_shape, n_pages: int, buf: torch.Tensor):
        self.shape, self.n_pages, self.buf = shape, n_pages, _need(buf, "buf", torch.uint8, (-1,))
        self.index = buf.get_device()
        self.rows = (shape.n_seqs, shape.q_len)
        self.ref = C.byref(shape)


class W4:
    """4-bit weight matrices laid out by rk_quant4."""

    def __init__(self, n_mat: int, n_out: int, k: int, group: int, codes: torch.Tensor, scales: torch.Tensor):
        self.n_mat, self.n_out, self.k, self.group = n_mat, n_out, k, group
        self.codes, self.scales = _need(codes, "codes", torch.uint8, None), _need(scales, "scales", torch.bfloat16, None)
        if codes.numel() < n_mat * n_out * k // 2 or scales.numel() < n_mat * n_out * (k // max(group, 1)):
            raise ValueError("codes or scales are too small for the shape")
        self.index = codes.get_device()
        self.struct = rk_w4(n_mat, n_out, k, group, _ptr(codes), _ptr(scales))
        self.ref = C.byref(self.struct)


class Q8:
    """Rows in 8 bits (rk_quant8's result, or codes and scales that a program keeps): codes int8 [n_mat, n_rows, k rounded
    up to a multiple of 16] (or [n_rows, ...] for one matrix), zeros behind k; scales float32 [n_mat, n_rows] or [n_rows]."""

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, k: int):
        shape = codes.shape
        if len(shape) not in (2, 3) or shape[-1] != (k + 15) // 16 * 16:
            raise ValueError(f"codes of k = {k} must be [n_mat, n_rows, {(k + 15) // 16 * 16}], not {tuple(shape)}")
        self._codes = _need(codes, "codes", torch.int8, None)
        self._scales = _need(scales, "scales", torch.float32, shape[:-1])
        self._set(shape[:-1], int(k), codes.get_device(), codes.device, _ptr(codes), _ptr(scales))

    def _set(self, rows, k, index, device, codes, scales):
        self.rows, self.k, self.index, self.device = rows, k, index, device
        self.n_mat, self.n_rows = (rows[0] if len(rows) == 2 else 1), rows[-1]
        self.struct = rk_q8(self.n_mat, self.n_rows, k, codes, scales)
        self.ref = C.byref(self.struct)

    @classmethod
    def _new(cls, rows, k: int, device: torch.device) -> "Q8":
        """For a call's own result: one allocation, of which codes and scales become views when somebody asks for them."""
        self = object.__new__(cls)
        at = 1
        for extent in rows:
            at *= extent
        self._split = at * ((k + 15) // 16 * 16)
        self._buf = _empty(self._split + 4 * at, torch.int8, device)
        self._codes = self._scales = None
        base = self._buf.data_ptr()
        self._set(rows, k, self._buf.get_device(), device, base, base + self._split)
        return self

    @property
    def codes(self) -> torch.Tensor:
        if self._codes is None:
            self._codes = self._buf[:self._split].view(self.rows + ((self.k + 15) // 16 * 16,))
        return self._codes

    @property
    def scales(self) -> torch.Tensor:
        if self._scales is None:
            self._scales = self._buf[self._split:].view(torch.float32).view(self.rows)
        return self._scales


def _rows(t: torch.Tensor, name: str, dtypes, width: int = -1) -> int:
    """Checks a matrix whose rows may be strided; the row stride in elements."""
    if t.dtype not in dtypes:
        raise TypeError(f"{name} must be {' or '.join(str(d) for d in dtypes)}, not {t.dtype}")
    _need(t, name, t.dtype, (-1, width), contiguous=False)
    if t.is_contiguous():
        return t.shape[1]
    if t.shape[0] > 0 and t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"the values of a row of {name} must be contiguous")
    if t.shape[0] > 1 and t.stride(0) < t.shape[1]:
        raise ValueError(f"the rows of {name} overlap")
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


_FLOATS = (torch.bfloat16, torch.float32)
_SCORES = {"softmax": 0, "sigmoid": 1}
_ROUTES = {}  # parameters of rk_moe_route as the C ABI takes them


def make_layout_struct(seg_off, seg_delta, seg_has_artifact):
    so = np.ascontiguousarray(seg_off, dtype=np.int64)
    sd = np.ascontiguousarray(seg_delta, dtype=np.int64)
    sh = np.ascontiguousarray(seg_has_artifact, dtype=np.uint8)
    lay = rk_layout(len(sd), so.ctypes.data_as(C.POINTER(C.c_int64)), sd.ctypes.data_as(C.POINTER(C.c_int64)),
                    sh.ctypes.data_as(C.POINTER(C.c_uint8)))
    return lay, (so, sd, sh)


def rk_check_request(seg_off, seg_delta, seg_has_artifact, prot_rows):
    """Host-only validation; returns (status, message)."""
    lay, keep = make_layout_struct(seg_off, seg_delta, seg_has_artifact)
    pr = np.ascontiguousarray(prot_rows, dtype=np.int32)
    msg = C.create_string_buffer(256)
    s = lib.rk_check_request(C.byref(lay), pr.ctypes.data_as(C.POINTER(C.c_int32)), len(pr), msg, 256)
    return s, msg.value.decode()


class Context:
    """rk_ctx: one per (device, head profile)."""

    def __init__(self, n_heads, n_groups, o_rank, d_model, global_heads, sm_scale, rope_base=10000.0,
                 group_size=8, d_latent=512, d_rope=64, d_v=128, value_phase=False):
        gh = np.ascontiguousarray(global_heads, dtype=np.int32)
        self._gh = gh
        self.profile = rk_profile(n_heads, n_groups, group_size, d_latent, d_rope, d_v, o_rank, d_model,
                                  float(sm_scale), float(rope_base), gh.ctypes.data_as(C.POINTER(C.c_int32)))
        self.handle = C.c_void_p()
        # value_phase: the output-phase variant (RK_VALUE_PHASE): attention outputs are 576 wide, W_uv [H,128,576]
        s = lib.rk_create_ex(C.byref(self.profile), 1 if value_phase else 0, C.byref(self.handle))
        if s != RK_OK:
            raise RKError(s, "rk_create failed")
        self.value_phase = bool(value_phase)
        self.ow = 576 if value_phase else 512
        self.n_heads, self.n_groups, self.n_local = n_heads, n_groups, n_heads - n_groups
        self.o_rank, self.d_model = o_rank, d_model

    @classmethod
    def from_profile(cls, p, value_phase=False):
        return cls(p.n_heads, p.n_groups, p.o_rank, p.d_model, p.global_heads, p.sm_scale, p.rope_base,
                   value_phase=value_phase)

    def check(self, s: int):
        if s != RK_OK:
            raise RKError(s, lib.rk_last_error(self.handle).decode())

    def close(self):
        if self.handle:
            lib.rk_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def rk_poll_status(self):
        self.check(lib.rk_poll_status(self.handle, _stream()))

    def rk_set_wait_limit_ms(self, ms: int):
        self.check(lib.rk_set_wait_limit_ms(self.handle, ms))

    def rk_check_selftest(self):
        self.check(lib.rk_check_selftest(self.handle, _stream()))

    def rk_test_starve_loads(self, on: int):
        self.check(lib.rk_test_starve_loads(self.handle, int(on)))

    def rk_request_create(self, seg_off, seg_delta, seg_has_artifact, prot_rows) -> "Request":
        return Request(self, seg_off, seg_delta, seg_has_artifact, prot_rows)

    # -- the five calls ---------------------------------------------------------------------
    def rk_relocate_q(self, req, q_rope_view: torch.Tensor, seg_begin: int, seg_end: int,
                      out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """q_rope_view: [n_rows, n_heads, 64] bf16 view (may be a strided slice of a wider tensor)."""
        n_rows, n_heads, w = q_rope_view.shape
        assert w == 64 and q_rope_view.stride(2) == 1 and q_rope_view.dtype == torch.bfloat16
        if out is None:
            out = _empty((seg_end - seg_begin, n_rows, n_heads, 64), dtype=torch.bfloat16,
                              device=q_rope_view.device)
        self.check(lib.rk_relocate_q(self.handle, req.handle, q_rope_view.data_ptr(), n_rows, n_heads,
                                     q_rope_view.stride(0), q_rope_view.stride(1), seg_begin, seg_end,
                                     out.data_ptr(), _stream()))
        return out

    def rk_mla_online_attn(self, req, kv, q_g, q_l, O_g=None, lse_g=None, O_l=None, lse_l=None):
        dev = kv.device
        if q_g is not None and O_g is None:
            O_g = _empty((req.T, self.n_groups, self.ow), dtype=torch.bfloat16, device=dev)
            lse_g = _empty((req.T, self.n_groups), dtype=torch.float32, device=dev)
        if q_l is not None and O_l is None:
            O_l = _empty((req.A, self.n_local, self.ow), dtype=torch.bfloat16, device=dev)
            lse_l = _empty((req.A, self.n_local), dtype=torch.float32, device=dev)
        self.check(lib.rk_mla_online_attn(self.handle, req.handle, _ptr(kv), _ptr(q_g), _ptr(q_l), _ptr(O_g),
                                          _ptr(lse_g), _ptr(O_l), _ptr(lse_l), _stream()))
        return O_g, lse_g, O_l, lse_l

    def rk_segmented_merge(self, O_part: torch.Tensor, lse_part: torch.Tensor, O=None, lse=None):
        P, n_rows, n_heads, d = O_part.shape
        assert d == 512 and lse_part.shape == (P, n_rows, n_heads) and lse_part.dtype == torch.float32
        dt = {torch.bfloat16: 0, torch.float32: 1}[O_part.dtype]
        if O is None:
            O = _empty((n_rows, n_heads, 512), dtype=torch.bfloat16, device=O_part.device)
            lse = _empty((n_rows, n_heads), dtype=torch.float32, device=O_part.device)
        self.check(lib.rk_segmented_merge(self.handle, P, n_rows, n_heads, _ptr(O_part), dt, _ptr(lse_part),
                                          _ptr(O), _ptr(lse), _stream()))
        return O, lse

    def rk_segmented_merge_phase(self, req, seg_begin: int, O_part: torch.Tensor, lse_part: torch.Tensor,
                                 row_pos: Optional[torch.Tensor] = None, O=None, lse=None):
        """Output-phase merge: part j belongs to segment seg_begin + j; O_part [P, n_rows, n_heads, 576]."""
        P, n_rows, n_heads, d = O_part.shape
        assert d == 576 and lse_part.shape == (P, n_rows, n_heads) and lse_part.dtype == torch.float32
        assert row_pos is None or (row_pos.dtype == torch.int32 and row_pos.shape == (n_rows,))
        dt = {torch.bfloat16: 0, torch.float32: 1}[O_part.dtype]
        if O is None:
            O = _empty((n_rows, n_heads, 576), dtype=torch.bfloat16, device=O_part.device)
            lse = _empty((n_rows, n_heads), dtype=torch.float32, device=O_part.device)
        self.check(lib.rk_segmented_merge_phase(self.handle, req.handle, seg_begin, P, n_rows, n_heads, _ptr(O_part), dt,
                                                _ptr(lse_part), _ptr(row_pos), _ptr(O), _ptr(lse), _stream()))
        return O, lse

    def rk_group_sliced_proj(self, req, O_g, O_l, W_uv, W_a, z_on_g=None, z_on_l=None, workspace=None):
        dev = W_uv.device
        width = self.n_groups * self.o_rank
        if O_g is not None and z_on_g is None:
            z_on_g = _empty((req.T, width), dtype=torch.bfloat16, device=dev)
        if O_l is not None and z_on_l is None:
            z_on_l = _empty((req.A, width), dtype=torch.bfloat16, device=dev)
        if workspace is None:
            workspace = _empty(max(req.workspace_bytes, 256), dtype=torch.uint8, device=dev)
        self.check(lib.rk_group_sliced_proj(self.handle, req.handle, _ptr(O_g), _ptr(O_l), _ptr(W_uv), _ptr(W_a),
                                            _ptr(z_on_g), _ptr(z_on_l), _ptr(workspace), workspace.numel(),
                                            _stream()))
        return z_on_g, z_on_l

    def rk_group_sliced_proj_static(self, req, O_g, O_l, W_uv, W_a, z_on_g, z_on_l):
        """Projection for callers that cannot allocate: outputs are passed in, the intermediate
        lives in the library's built-in 32 MiB array (shared by all calls; see include/rk.h)."""
        self.check(lib.rk_group_sliced_proj_static(self.handle, req.handle, _ptr(O_g), _ptr(O_l), _ptr(W_uv),
                                                   _ptr(W_a), _ptr(z_on_g), _ptr(z_on_l), _stream()))
        return z_on_g, z_on_l

    def rk_protected_rows(self, seg_off, seg_delta, seg_has_artifact, dirty_rows=None, scores=None, *, edge_rows=128,
                          tail_rows=32768, budget_bp=0, device="cuda", out=None, workspace=None):
        """Eq. (protected) on the device.  Returns (rows_out, count_out): a device int32 buffer of capacity T
        whose first count_out[0] entries are the ascending protected rows, and the device int64 count.
        Nothing is synchronised; `protected_rows_to_host` reads the list back."""
        lay, keep = make_layout_struct(seg_off, seg_delta, seg_has_artifact)
        pol = rk_policy(int(edge_rows), int(tail_rows), int(budget_bp))
        T, S = int(keep[0][-1]), len(keep[1])
        if workspace is None:
            need = C.c_size_t(0)
            s = lib.rk_protected_rows_workspace_bytes(T, S, C.byref(need))
            if s != 0:
                raise RKError(s, "rk_protected_rows_workspace_bytes")
            workspace = _empty(need.value, dtype=torch.uint8, device=device)
        if out is None:
            out = (_empty(T, dtype=torch.int32, device=device), _empty(1, dtype=torch.int64, device=device))
        n_dirty = 0 if dirty_rows is None else dirty_rows.numel()
        self.check(lib.rk_protected_rows(self.handle, C.byref(lay), C.byref(pol), _ptr(dirty_rows), n_dirty, _ptr(scores),
                                         _ptr(out[0]), _ptr(out[1]), _ptr(workspace), workspace.numel(), _stream()))
        return out

    @staticmethod
    def protected_rows_to_host(out) -> np.ndarray:
        n = int(out[1].item())
        return out[0][:n].cpu().numpy()

    def rk_moe_fanout(self, p: torch.Tensor, tau: float, fence: bool = False, k_out=None, keep_out=None):
        """Eq. (moe): p [n, 6] float32 Top-6 router weights -> (K_t [n] uint8, keep mask [n] uint8)."""
        assert p.dtype == torch.float32 and p.dim() == 2 and p.shape[1] == 6 and p.is_contiguous()
        n = p.shape[0]
        if k_out is None:
            k_out = _empty(n, dtype=torch.uint8, device=p.device)
            keep_out = _empty(n, dtype=torch.uint8, device=p.device)
        self.check(lib.rk_moe_fanout(self.handle, _ptr(p), n, float(tau), int(bool(fence)), _ptr(k_out), _ptr(keep_out),
                                     _stream()))
        return k_out, keep_out

    def rk_combine_offline(self, req, z_on_g, z_on_l, z_off, W_b, z=None, y=None):
        dev = z_on_g.device
        if z is None:
            z = _empty((req.T, self.n_groups * self.o_rank), dtype=torch.bfloat16, device=dev)
        if W_b is not None and y is None:
            y = _empty((req.T, self.d_model), dtype=torch.bfloat16, device=dev)
        self.check(lib.rk_combine_offline(self.handle, req.handle, _ptr(z_on_g), _ptr(z_on_l), _ptr(z_off),
                                          _ptr(W_b), _ptr(z), _ptr(y), _stream()))
        return z, y

    def rk_mla_off_build(self, req, kv, row_begin, row_end, q_l_rows, W_uv, W_a, z_off_rows=None, workspace=None):
        """Offline artifact rows [row_begin, row_end): documents alone at position zero, Local heads."""
        n = row_end - row_begin
        if z_off_rows is None:
            z_off_rows = _empty((n, self.n_groups * self.o_rank), dtype=torch.bfloat16, device=kv.device)
        ws = C.c_size_t()
        self.check(lib.rk_mla_off_workspace_bytes(req.handle, n, C.byref(ws)))
        if workspace is None:
            workspace = _empty(max(ws.value, 256), dtype=torch.uint8, device=kv.device)
        self.check(lib.rk_mla_off_build(self.handle, req.handle, _ptr(kv), row_begin, row_end, _ptr(q_l_rows),
                                        _ptr(W_uv), _ptr(W_a), _ptr(z_off_rows), _ptr(workspace), workspace.numel(),
                                        _stream()))
        return z_off_rows

    # -- decode -------------------------------------------------------------------------------
    def rk_cache4_append(self, pages: torch.Tensor, table: CacheTable, c: torch.Tensor, k_rope: torch.Tensor,
                         new_off: torch.Tensor):
        """Rows new_off[s] .. new_off[s+1] of c [n, 512] and k_rope [n, 64] (before rotation) become the last rows of
        segment s; table.seg_len already counts them.  pages: uint8 [n_pages, 26624].  Rows may be strided."""
        n = c.shape[0]
        n_pages = _pages(pages)
        _here(table, "table")
        _need(c, "c", torch.bfloat16, (-1, 512), contiguous=False)
        _need(k_rope, "k_rope", torch.bfloat16, (n, 64), contiguous=False)
        _need(new_off, "new_off", torch.int32, (table.n_segs + 1,))
        c_stride, r_stride = 512, 64  # a single row's stride is arbitrary and never used
        if not (c.is_contiguous() and k_rope.is_contiguous()) and n > 0:
            if c.stride(1) != 1 or k_rope.stride(1) != 1:
                raise ValueError("the values of a row of c and k_rope must be contiguous")
            if n > 1:
                c_stride, r_stride = c.stride(0), k_rope.stride(0)
        s = lib.rk_cache4_append(self.handle, pages.data_ptr(), n_pages, table.ref, c.data_ptr(), c_stride, k_rope.data_ptr(),
                                 r_stride, new_off.data_ptr(), n, _quick_stream())
        if s:
            self.check(s)

    def rk_cache4_read(self, pages: torch.Tensor, table: CacheTable, row_off: torch.Tensor, n_rows: int, kv=None) -> torch.Tensor:
        """The last row_off[s+1] - row_off[s] rows of every segment s as packed bf16 rows kv [n_rows, 576]; rows from
        row_off[n_segs] on are left as they were."""
        n_pages = _pages(pages)
        _here(table, "table")
        _need(row_off, "row_off", torch.int32, (table.n_segs + 1,))
        if kv is None:
            kv = _empty((n_rows, 576), torch.bfloat16, pages.device)
        else:
            _need(kv, "kv", torch.bfloat16, (n_rows, 576))
        s = lib.rk_cache4_read(self.handle, pages.data_ptr(), n_pages, table.ref, row_off.data_ptr(), n_rows, kv.data_ptr(),
                               _quick_stream())
        if s:
            self.check(s)
        return kv

    def rk_decode_plan(self, table: CacheTable, n_pages: int, seq_off: torch.Tensor, item_seg: torch.Tensor,
                       item_delta: torch.Tensor, q_pos: torch.Tensor, *, max_tiles: int, plan: Optional[DecodePlan] = None) -> DecodePlan:
        """Work list of a decode step: request b sees the segments item_seg[seq_off[b]:seq_off[b+1]] at the request offsets
        item_delta; q_pos [n_seqs, q_len] are its query tokens' positions.  max_tiles bounds the sum over the items of
        ceil(rows / 128).  With plan= its buffer is filled anew (a captured graph keeps using it)."""
        _here(table, "table")
        if plan is not None:
            _here(plan, "plan")
        _need(q_pos, "q_pos", torch.int32, (-1, -1))
        _need(seq_off, "seq_off", torch.int32, (q_pos.shape[0] + 1,))
        _need(item_seg, "item_seg", torch.int32, (-1,))
        _need(item_delta, "item_delta", torch.int32, (item_seg.numel(),))
        shape = rk_decode_shape(q_pos.shape[0], q_pos.shape[1], item_seg.numel(), int(max_tiles))
        need = C.c_size_t(0)
        self.check(lib.rk_decode_plan_bytes(self.handle, C.byref(shape), C.byref(need)))
        if plan is None:
            plan = DecodePlan(shape, int(n_pages), _empty(need.value, dtype=torch.uint8, device=q_pos.device))
        else:
            plan.__init__(shape, int(n_pages), plan.buf)
        self.check(lib.rk_decode_plan(self.handle, C.byref(shape), table.ref, int(n_pages), _ptr(seq_off), _ptr(item_seg),
                                      _ptr(item_delta), _ptr(q_pos), _ptr(plan.buf), plan.buf.numel(), _quick_stream()))
        return plan

    def rk_cache4_attn(self, pages: torch.Tensor, plan: DecodePlan, q: torch.Tensor, O=None, lse=None, workspace=None):
        """q [n_seqs, q_len, n_heads, 576] -> (O [n_seqs, q_len, n_heads, 512] bf16, lse fp32)."""
        rows = plan.rows + (self.n_heads,)
        n_pages = _pages(pages)
        _here(plan, "plan")
        _need(q, "q", torch.bfloat16, rows + (576,))
        device = q.device
        if O is None:
            O = _empty(rows + (512,), torch.bfloat16, device)
        else:
            _need(O, "O", torch.bfloat16, rows + (512,))
        if lse is None:
            lse = _empty(rows, torch.float32, device)
        else:
            _need(lse, "lse", torch.float32, rows)
        if workspace is None:
            need = C.c_size_t(0)
            self.check(lib.rk_cache4_attn_workspace_bytes(self.handle, plan.ref, C.byref(need)))
            size = need.value
            workspace = _empty(size, torch.uint8, device)
        else:
            _need(workspace, "workspace", torch.uint8, (-1,))
            size = workspace.numel()
        buf = plan.buf
        s = lib.rk_cache4_attn(self.handle, plan.ref, buf.data_ptr(), buf.numel(), pages.data_ptr(), n_pages, q.data_ptr(),
                               O.data_ptr(), lse.data_ptr(), workspace.data_ptr(), size, _quick_stream())
        if s:
            self.check(s)
        return O, lse

    def rk_quant4(self, w: torch.Tensor, group: int, w4: Optional[W4] = None) -> W4:
        """Lays out w [n_mat, n_out, k] bf16 as 4-bit codes with one bf16 scale per `group` columns of a row."""
        _need(w, "w", torch.bfloat16, (-1, -1, -1))
        n_mat, n_out, k = w.shape
        if w4 is None:
            n = w.numel()
            w4 = W4(n_mat, n_out, k, int(group), _empty(max(n // 2, 16), dtype=torch.uint8, device=w.device),
                    _empty(max(n // max(int(group), 1), 8), dtype=torch.bfloat16, device=w.device))
        elif (w4.n_mat, w4.n_out, w4.k, w4.group) != (n_mat, n_out, k, int(group)):
            raise ValueError("w4 has another shape")
        _here(w4, "w4")
        self.check(lib.rk_quant4(self.handle, _ptr(w), w4.ref, _quick_stream()))
        return w4

    def rk_matvec4(self, w4: W4, x: torch.Tensor, y: Optional[torch.Tensor] = None, out_dtype=torch.bfloat16) -> torch.Tensor:
        """x [n_tok, n_mat, k] bf16 (tokens may be strided) -> y [n_tok, n_mat, n_out], bf16 or float32."""
        n, n_mat, n_out, k = x.shape[0], w4.n_mat, w4.n_out, w4.k
        _here(w4, "w4")
        _need(x, "x", torch.bfloat16, (n, n_mat, k), contiguous=False)
        if y is not None:
            out_dtype = y.dtype
        if out_dtype is not torch.bfloat16 and out_dtype is not torch.float32:
            raise TypeError(f"the products' outputs are bfloat16 or float32, not {out_dtype}")
        if y is None:
            y = _empty((n, n_mat, n_out), out_dtype, x.device)
        else:
            _need(y, "y", out_dtype, (n, n_mat, n_out), contiguous=False)
        x_stride, y_stride = n_mat * k, n_mat * n_out
        if not (x.is_contiguous() and y.is_contiguous()) and n > 0:
            for t, name in ((x, "x"), (y, "y")):
                if not t[0].is_contiguous():
                    raise ValueError(f"the values of a token of {name} must be contiguous")
            if n > 1:
                x_stride, y_stride = x.stride(0), y.stride(0)
        dt = 0 if out_dtype is torch.bfloat16 else 1
        s = lib.rk_matvec4(self.handle, w4.ref, x.data_ptr(), x_stride, n, y.data_ptr(), y_stride, dt, _quick_stream())
        if s:
            self.check(s)
        return y

    # -- behind the attention: experts and tokens -----------------------------------------------
    def rk_moe_route(self, logits: torch.Tensor, k: int, *, bias: Optional[torch.Tensor] = None, score: str = "softmax",
                     n_groups: int = 1, top_groups: int = 1, group_top: int = 1, renorm: bool = False, scale: float = 1.0,
                     ids=None, weights=None):
        """logits [n, E] bf16 or float32 (rows may be strided) -> (ids [n, k] int32, weights [n, k] float32): the k experts of
        the largest score + bias among those of the top_groups best groups, in descending order."""
        stride = _rows(logits, "logits", _FLOATS)
        n, n_experts = logits.shape
        if score not in _SCORES:
            raise ValueError(f"score must be 'softmax' or 'sigmoid', not {score!r}")
        if bias is not None:
            _need(bias, "bias", torch.float32, (n_experts,))
        if ids is None:
            ids = _empty((n, k), torch.int32, logits.device)
        else:
            _need(ids, "ids", torch.int32, (n, k))
        if weights is None:
            weights = _empty((n, k), torch.float32, logits.device)
        else:
            _need(weights, "weights", torch.float32, (n, k))
        key = (n_experts, k, n_groups, top_groups, group_top, score, renorm, scale)
        route = _ROUTES.get(key)
        if route is None:  # (a program has a few of them: one per kind of layer)
            if len(_ROUTES) > 64:
                _ROUTES.clear()
            route = _ROUTES[key] = rk_route(n_experts, k, n_groups, top_groups, group_top, _SCORES[score], 1 if renorm else 0, scale)
        s = lib.rk_moe_route(self.handle, C.byref(route), logits.data_ptr(), 0 if logits.dtype is torch.bfloat16 else 1, stride,
                             None if bias is None else bias.data_ptr(), n, ids.data_ptr(), weights.data_ptr(), _quick_stream())
        if s:
            self.check(s)
        return ids, weights

    def rk_moe_group(self, ids: torch.Tensor, n_experts: int, keep: Optional[torch.Tensor] = None, row_off=None, rows=None):
        """ids [n, k] int32 (and keep [n] uint8, rk_moe_fanout's masks) -> (row_off [n_experts + 1], rows [n * k]) int32: the
        pairs t * k + s by expert; the places behind the last listed pair hold -1."""
        _need(ids, "ids", torch.int32, (-1, -1))
        n, k = ids.shape
        if keep is not None:
            _need(keep, "keep", torch.uint8, (n,))
        if row_off is None:
            row_off = _empty(n_experts + 1, torch.int32, ids.device)
        else:
            _need(row_off, "row_off", torch.int32, (n_experts + 1,))
        if rows is None:
            rows = _empty(n * k, torch.int32, ids.device)
        else:
            _need(rows, "rows", torch.int32, (n * k,))
        s = lib.rk_moe_group(self.handle, ids.data_ptr(), None if keep is None else keep.data_ptr(), n, k, n_experts,
                             row_off.data_ptr(), rows.data_ptr(), _quick_stream())
        if s:
            self.check(s)
        return row_off, rows

    def rk_quant8(self, x: torch.Tensor, q8: Optional[Q8] = None) -> Q8:
        """Rows of x in 8 bits with a scale each: x [n, k] bf16 (rows may be strided), or [n_mat, n, k] contiguous (weights)."""
        if x.dim() == 3:
            _need(x, "x", torch.bfloat16, (-1, -1, -1))
            stride = x.shape[2]
        else:
            stride = _rows(x, "x", (torch.bfloat16,))
        k = x.shape[-1]
        if q8 is None:
            q8 = Q8._new(tuple(x.shape[:-1]), k, x.device)
        else:
            _here(q8, "q8")
            if (q8.n_mat, q8.n_rows, q8.k) != (x.shape[0] if x.dim() == 3 else 1, x.shape[-2], k):
                raise ValueError("q8 has another shape")
        s = lib.rk_quant8(self.handle, x.data_ptr(), stride, q8.ref, _quick_stream())
        if s:
            self.check(s)
        return q8

    def _out8(self, w: Q8, x: Q8, n: int, y, out_dtype):
        """Output of an 8-bit product: tensor, row stride, type number."""
        _here(w, "w")
        _here(x, "x")
        if y is not None:
            out_dtype = y.dtype
        if out_dtype is not torch.bfloat16 and out_dtype is not torch.float32:
            raise TypeError(f"the products' outputs are bfloat16 or float32, not {out_dtype}")
        stride = w.n_rows
        if y is None:
            y = _empty((n, stride), out_dtype, x.device)
        else:
            stride = _rows(y, "y", _FLOATS, w.n_rows)
            if y.shape[0] != n:
                raise ValueError(f"y must have {n} rows, not {y.shape[0]}")
        return y, stride, 0 if out_dtype is torch.bfloat16 else 1

    def rk_matmul8(self, w: Q8, x: Q8, y: Optional[torch.Tensor] = None, out_dtype=torch.bfloat16) -> torch.Tensor:
        """y [n, n_out] = x w^T of 8-bit rows, bf16 or float32 (rows of y may be strided)."""
        y, stride, dt = self._out8(w, x, x.n_rows, y, out_dtype)
        s = lib.rk_matmul8(self.handle, w.ref, x.ref, y.data_ptr(), stride, dt, _quick_stream())
        if s:
            self.check(s)
        return y

    def rk_matmul8_experts(self, w: Q8, x: Q8, row_off: torch.Tensor, rows: torch.Tensor, per: int,
                           y: Optional[torch.Tensor] = None, out_dtype=torch.bfloat16) -> torch.Tensor:
        """y[p] = w[e] x[p // per] for the pairs p = rows[row_off[e]:row_off[e + 1]] of every expert e (rk_moe_group's lists);
        rows of y that no list names are left as they were."""
        _need(row_off, "row_off", torch.int32, (w.n_mat + 1,))
        _need(rows, "rows", torch.int32, (-1,))
        n = rows.shape[0]
        y, stride, dt = self._out8(w, x, n, y, out_dtype)
        s = lib.rk_matmul8_experts(self.handle, w.ref, x.ref, row_off.data_ptr(), rows.data_ptr(), n, per, y.data_ptr(), stride, dt,
                                   _quick_stream())
        if s:
            self.check(s)
        return y

    def rk_sample(self, logits: torch.Tensor, u: torch.Tensor, *, temperature=None, top_k=None, top_p=None, min_p=None, tokens=None,
                  probs=None):
        """One token per row of logits [n, vocab] (bf16 or float32, rows may be strided) from the uniform random numbers u [n];
        temperature, top_p, min_p float32 [n], top_k int32 [n], each None for off.  Returns (tokens [n] int32, probs [n])."""
        stride = _rows(logits, "logits", _FLOATS)
        n, vocab = logits.shape
        _need(u, "u", torch.float32, (n,))
        ptrs = []
        for t, name, dtype in ((temperature, "temperature", torch.float32), (top_k, "top_k", torch.int32),
                               (top_p, "top_p", torch.float32), (min_p, "min_p", torch.float32)):
            ptrs.append(None if t is None else _need(t, name, dtype, (n,)).data_ptr())
        if tokens is None:
            tokens = _empty((n,), torch.int32, logits.device)
        else:
            _need(tokens, "tokens", torch.int32, (n,))
        if probs is None:
            probs = _empty((n,), torch.float32, logits.device)
        else:
            _need(probs, "probs", torch.float32, (n,))
        s = lib.rk_sample(self.handle, logits.data_ptr(), 0 if logits.dtype is torch.bfloat16 else 1, stride, n, vocab, u.data_ptr(),
                          *ptrs, tokens.data_ptr(), probs.data_ptr(), _quick_stream())
        if s:
            self.check(s)
        return tokens, probs

    def alloc_layer_buffers(self, req, device) -> dict:
        G, L, T, A = self.n_groups, self.n_local, req.T, req.A
        width = G * self.o_rank
        bf, f32 = torch.bfloat16, torch.float32
        e = lambda shape, dt=bf: _empty(shape, dtype=dt, device=device)
        return dict(kv=e((T, 576)), q_g=e((T, G, 576)), q_l=e((max(A, 1), L, 576)),
                    z_off=e((max(req.n_off_rows, 1), width)), O_g=e((T, G, self.ow)), O_l=e((max(A, 1), L, self.ow)),
                    z_on_g=e((T, width)), z_on_l=e((max(A, 1), width)), z=e((T, width)), y=e((T, self.d_model)),
                    lse_g=e((T, G), f32), lse_l=e((max(A, 1), L), f32),
                    workspace=_empty(max(req.workspace_bytes, 256), dtype=torch.uint8, device=device))

    def rk_layer_host(self, req, kv_h, q_g_h, q_l_h, z_off_h, W_uv, W_a, W_b, bufs: dict, y_h: torch.Tensor):
        """Whole layer from pinned host tensors: H2D copies, the three device calls, D2H of y, sync."""
        b = rk_layer_buffers(*[bufs[n].data_ptr() for n in ("kv", "q_g", "q_l", "z_off", "O_g", "O_l", "z_on_g",
                                                            "z_on_l", "z", "y", "lse_g", "lse_l", "workspace")],
                             bufs["workspace"].numel())
        self.check(lib.rk_layer_host(self.handle, req.handle, _ptr(kv_h), _ptr(q_g_h), _ptr(q_l_h), _ptr(z_off_h),
                                     _ptr(W_uv), _ptr(W_a), _ptr(W_b), C.byref(b), _ptr(y_h), _stream()))
        return y_h


def _buffers_struct(bufs: dict) -> rk_layer_buffers:
    return rk_layer_buffers(*[bufs[n].data_ptr() for n in ("kv", "q_g", "q_l", "z_off", "O_g", "O_l", "z_on_g", "z_on_l",
                                                           "z", "y", "lse_g", "lse_l", "workspace")],
                            bufs["workspace"].numel())


def rk_layer_stack_host(ctx: "Context", layers, bufs0: dict, bufs1: dict):
    """layers: list of dicts with keys req, kv, q_g, q_l, z_off (pinned host tensors), W_uv, W_a, W_b (device
    tensors) and y (pinned host output).  Runs the stack with cross-layer prefetch."""
    arr = (rk_layer_io * len(layers))()
    for i, l in enumerate(layers):
        arr[i] = rk_layer_io(l["req"].handle.value, _ptr(l["kv"]), _ptr(l["q_g"]), _ptr(l["q_l"]), _ptr(l["z_off"]),
                             _ptr(l["W_uv"]), _ptr(l["W_a"]), _ptr(l["W_b"]), _ptr(l["y"]))
    b0, b1 = _buffers_struct(bufs0), _buffers_struct(bufs1)
    ctx.check(lib.rk_layer_stack_host(ctx.handle, len(layers), arr, C.byref(b0), C.byref(b1), _stream()))


class Request:
    """rk_request: validated geometry of one request + protected-row list."""

    def __init__(self, ctx: Context, seg_off, seg_delta, seg_has_artifact, prot_rows):
        self.ctx = ctx
        lay, keep = make_layout_struct(seg_off, seg_delta, seg_has_artifact)
        pr = np.ascontiguousarray(prot_rows, dtype=np.int32)
        self.handle = C.c_void_p()
        ctx.check(lib.rk_request_create(ctx.handle, C.byref(lay), pr.ctypes.data_as(C.POINTER(C.c_int32)), len(pr),
                                        C.byref(self.handle)))
        info = rk_request_info()
        ctx.check(lib.rk_request_get_info(self.handle, C.byref(info)))
        self.T, self.A, self.n_off_rows = info.n_rows, info.n_prot, info.n_off_rows
        self.pairs_global, self.pairs_local = info.pairs_global, info.pairs_local
        self.n_tiles_global, self.n_tiles_local = info.n_tiles_global, info.n_tiles_local
        ws = C.c_size_t()
        ctx.check(lib.rk_workspace_bytes(self.handle, C.byref(ws)))
        self.workspace_bytes = ws.value

    def close(self):
        if self.handle:
            lib.rk_request_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
