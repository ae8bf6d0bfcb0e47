"""ctypes binding of ``liblr_verify.so`` with the names of the C ABI.

Argument marshalling only: every step of the verify pass runs in the CUDA
kernels behind ``lr_verify_attention``, ``lr_accept_greedy`` and ``lr_commit``.
torch is used for device memory and streams.  There is no fallback: if the
library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from typing import Optional

import numpy as np
import torch

from .build import LIB_PATH

LR_OK = 0
STATUS_NAMES = {0: "LR_OK", -1: "LR_EINVAL", -2: "LR_EUNSUPPORTED", -3: "LR_ECUDA", -4: "LR_ETIMEOUT", -5: "LR_EBOUNDS",
                -6: "LR_ENOMEM"}

KV_BF16, KV_FP8, KV_FP4 = 0, 1, 2  # LR_KV_*
PATH_AUTO, PATH_GENERIC, PATH_TENSOR_CORE, PATH_PAIR = 0, 1, 2, 3
ACCEPT_STATIC_MAX_ROWS = 4096  # LR_ACCEPT_STATIC_MAX_ROWS
COMMIT_MAX_REQUESTS = 4096  # LR_COMMIT_MAX_REQUESTS
COMPACT_MAX_REQUESTS = 8192  # LR_COMPACT_MAX_REQUESTS


class LrError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str):
        self.status = status
        super().__init__(f"{where}: {STATUS_NAMES.get(status, status)}: {detail}")


class lr_model(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_q_heads", "n_kv_heads", "head_dim", "page_size", "vocab")]


class lr_batch(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_req", "n_branch", "n_span", "n_page_slots")] + [
        (n, C.c_void_p)  # int32 arrays
        for n in ("req_span_off", "span_len", "span_slot", "br_req", "br_depth", "br_own_len", "br_own_slot",
                  "br_n_draft", "cu_q", "page_ids")
    ] + [("n_pool_pages", C.c_int64), ("seg_parent", C.c_void_p)]


class lr_cycle_stats(C.Structure):
    _fields_ = [(n, C.c_int64) for n in ("stages", "steps", "time", "verdicts_used", "peak_in_flight")]


class lr_plan_info(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("tensor_core_ok", "path", "uses_tensor_core", "n_cta", "n_pieces",
                                         "n_merge_targets", "n_partial_slots")]


class lr_partition_info(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_cta", "n_merge_targets", "n_partial_slots")] + [("longest_load", C.c_int64)]


class lr_fp8_cache(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("k_d", "v_d", "k_scale_d", "v_scale_d")] + [("n_pages", C.c_int64)]


class lr_fp4_cache(C.Structure):
    _fields_ = lr_fp8_cache._fields_


class lr_kv_cache(C.Structure):
    _fields_ = [("kind", C.c_int32)] + lr_fp8_cache._fields_


class lr_rope_spec(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("rot_dim", "interleaved", "scaling")] + [(n, C.c_double) for n in ("base", "factor", "original", "lo", "hi", "amplitude")]


class lr_pass_host_io(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in (
        "q_h", "logits_h", "draft_ids_h", "verdict_h", "out_h", "n_accept_h", "bonus_id_h", "n_steps_accepted_h",
        "survivor_h", "committed_len_h", "keep_off_h", "free_off_h", "keep_pages_h", "keep_valid_h", "free_pages_h")]


_lib = None


def lib() -> C.CDLL:
    """The loaded C-ABI library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2506_19830_b200.build` "
                "(there is no fallback implementation)")
        L = C.CDLL(LIB_PATH)
        vp, i32, i64, f32, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_size_t
        sig = {
            "lr_validate_batch": [C.POINTER(lr_model), C.POINTER(lr_batch)],
            "lr_create": [C.POINTER(vp), C.POINTER(lr_model), C.c_int],
            "lr_destroy": [vp],
            "lr_plan_bytes": [vp, C.POINTER(lr_batch), C.POINTER(sz)],
            "lr_plan_create": [vp, C.POINTER(lr_batch), vp, sz, vp, C.POINTER(vp)],
            "lr_plan_begin": [vp, C.POINTER(lr_batch), C.POINTER(sz), C.POINTER(vp)],
            "lr_plan_finish": [vp, vp, sz, vp, C.POINTER(vp)],
            "lr_plan_drop": [vp],
            "lr_plan_destroy": [vp],
            "lr_plan_set_attention_path": [vp, C.c_int],
            "lr_plan_describe": [vp, C.POINTER(lr_plan_info)],
            "lr_debug_partitions": [C.POINTER(lr_model), C.POINTER(lr_batch), i32, C.POINTER(lr_partition_info), C.POINTER(lr_partition_info),
                                    C.POINTER(i32)],
            "lr_plan_debug_set_page": [vp, i32, i32, vp],
            "lr_plan_debug_set_wait_limit": [vp, C.c_uint32],
            "lr_plan_debug_set_phantom_bytes": [vp, C.c_uint32],
            "lr_verify_attention": [vp, vp, vp, vp, vp, vp, f32, vp],
            "lr_accept_scratch_bytes": [i32, C.POINTER(sz)],
            "lr_accept_greedy": [vp, vp, i64, vp, vp, i32, i32, vp, vp, vp, vp, vp],
            "lr_accept_greedy_static": [vp, vp, i64, vp, vp, i32, i32, vp, vp, vp, vp],
            "lr_accept_sample_scratch_bytes": [vp, i32, C.POINTER(sz)],
            "lr_accept_sample": [vp, vp, i64, vp, vp, i32, i32, f32, vp, vp, vp, vp, vp, vp, vp],
            "lr_accept_sample_filtered_scratch_bytes": [vp, i32, C.POINTER(sz)],
            "lr_accept_sample_filtered": [vp, vp, i64, vp, vp, i32, i32, f32, i32, f32, vp, vp, vp, vp, vp, vp, vp, vp],
            "lr_accept_sample_drafted_scratch_bytes": [vp, i32, C.POINTER(sz)],
            "lr_accept_sample_drafted": [vp, vp, i64, vp, i64, vp, vp, i32, i32, f32, f32, vp, vp, vp, vp, vp, vp, vp, vp],
            "lr_commit": [vp] + [vp] * 10 + [vp],
            "lr_cycle_simulate_sync": [i32, i64, i64, vp, i64, C.POINTER(lr_cycle_stats)],
            "lr_cycle_simulate_async": [i32, i64, i64, vp, i64, C.POINTER(lr_cycle_stats)],
            "lr_cycle_best_strategy": [i32, C.c_double, C.c_double, C.c_double, C.c_double, i32, C.POINTER(i32),
                                       C.POINTER(i32), C.POINTER(C.c_double)],
            "lr_compact_scratch_bytes": [vp, C.POINTER(sz)],
            "lr_compact": [vp] * 10,
            "lr_fp8_write": [vp, vp, vp, i64, vp, i64, vp, i32, vp, vp],
            "lr_fp8_read": [vp, vp, vp, i32, vp, i64, vp, i64, vp, vp],
            "lr_verify_attention_fp8": [vp, vp, vp, vp, vp, f32, vp],
            "lr_compact_fp8": [vp] * 8,
            "lr_fp4_write": [vp, vp, vp, i64, vp, i64, vp, i32, vp, vp],
            "lr_fp4_read": [vp, vp, vp, i32, vp, i64, vp, i64, vp, vp],
            "lr_verify_attention_fp4": [vp, vp, vp, vp, vp, f32, vp],
            "lr_compact_fp4": [vp] * 8,
            "lr_rope_create": [C.POINTER(vp), C.POINTER(lr_rope_spec)],
            "lr_rope_destroy": [vp],
            "lr_rope_frequencies": [vp, vp, C.POINTER(C.c_double)],
            "lr_rope_write": [vp, vp, vp, vp, vp, i64, vp, vp, i64, vp, i64, vp, i32, vp, vp],
            "lr_copy_pages": [vp, vp, vp, i32, vp, vp, i32, vp, vp],
            "lr_pass_staging_bytes": [vp, C.POINTER(sz)],
            "lr_verify_pass": [vp, vp, C.c_char_p, f32, vp, vp],
            "lr_verify_pass_host": [vp, C.POINTER(lr_pass_host_io), vp, vp, vp, sz, f32, vp],
            "lr_poll_status": [vp, vp, C.POINTER(i32)],
        }
        for name, args in sig.items():
            fn = getattr(L, name)
            fn.argtypes = args
            fn.restype = C.c_int
        L.lr_launch_count.argtypes = [vp]
        L.lr_launch_count.restype = C.c_int64
        L.lr_cycle_speedup.argtypes = [i32, i32, C.c_double, C.c_double]
        L.lr_cycle_speedup.restype = C.c_double
        L.lr_strerror.argtypes = [C.c_int]
        L.lr_strerror.restype = C.c_char_p
        L.lr_last_error.argtypes = []
        L.lr_last_error.restype = C.c_char_p
        _lib = L
    return _lib


def _check(status: int, where: str):
    if status != LR_OK:
        raise LrError(status, where, lib().lr_last_error().decode(errors="replace"))


def _i32(a) -> np.ndarray:
    return np.ascontiguousarray(a, dtype=np.int32)


def _addr(a: np.ndarray) -> int:
    return a.__array_interface__["data"][0]


class HostBatch:
    """An ``lr_batch`` and the int32 host tables it points to, side by side in one array: asking numpy for an address takes a
    microsecond, and a serving loop makes a plan every cycle."""

    FIELDS = ("req_span_off", "span_len", "span_slot", "br_req", "br_depth", "br_own_len", "br_own_slot", "br_n_draft",
              "cu_q", "page_ids")

    def __init__(self, batch):
        tables = [_i32(getattr(batch, f)).ravel() for f in self.FIELDS]
        parent = getattr(batch, "seg_parent", None)  # tree of draft steps; absent = nested chain (NULL)
        if parent is not None:
            tables.append(_i32(parent).ravel())
        self.tables = np.concatenate(tables)
        n = [len(t) for t in tables]
        at = [_addr(self.tables)]
        for k in n[:-1]:
            at.append(at[-1] + 4 * k)
        self.c = lr_batch(n[0] - 1, n[3], n[1], n[9], *at[:10], int(batch.n_pool_pages), at[10] if parent is not None else None)


_PASS_IO = struct.Struct("23q").pack  # lr_pass_io


def _model_struct(model) -> lr_model:
    return lr_model(int(model.n_q_heads), int(model.n_kv_heads), int(model.head_dim), int(model.page_size),
                    int(model.vocab))


def lr_validate_batch(model, batch) -> None:
    hb = HostBatch(batch)
    m = _model_struct(model)
    _check(lib().lr_validate_batch(C.byref(m), C.byref(hb.c)), "lr_validate_batch")


def lr_debug_partitions(model, batch, n_sm: int):
    """(attention, pass, form of a small pass): how the attention work of a batch is split on a device of ``n_sm`` SMs."""
    hb, m, small = HostBatch(batch), _model_struct(model), C.c_int32()
    parts = [lr_partition_info(), lr_partition_info()]
    _check(lib().lr_debug_partitions(C.byref(m), C.byref(hb.c), n_sm, C.byref(parts[0]), C.byref(parts[1]), C.byref(small)),
           "lr_debug_partitions")
    attention, whole_pass = ({n: int(getattr(p, n)) for n, _ in p._fields_} for p in parts)
    return attention, whole_pass, small.value


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream_ptr(stream: Optional[torch.cuda.Stream]) -> int:
    # the raw handle of the current stream: building a torch.cuda.Stream object for it costs 3 us a call
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice()) if stream is None else stream.cuda_stream


def _stream_on(device: int, stream: Optional[torch.cuda.Stream]) -> int:
    """The stream given, or the current one of the context's device, which need not be the current device."""
    return torch._C._cuda_getCurrentRawStream(device) if stream is None else stream.cuda_stream


class Fp8Cache:
    """``lr_fp8_cache`` over four tensors of the caller's: codes [pages, KV heads, 16, head size] (``torch.float8_e4m3fn``) and scales
    [pages, KV heads, 16] (``torch.float8_e8m0fnu``), of K and of V; ``torch.uint8`` serves for either.  ``empty`` makes them."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor):
        shape = k.shape
        for t, want, kind in ((k, shape, torch.float8_e4m3fn), (v, shape, torch.float8_e4m3fn), (k_scale, shape[:3], torch.float8_e8m0fnu),
                              (v_scale, shape[:3], torch.float8_e8m0fnu)):
            if t.shape != want or len(shape) != 4 or shape[2] != 16 or t.dtype not in (kind, torch.uint8) or not t.is_contiguous() or t.device != k.device:
                raise ValueError(f"an 8-bit cache is codes [pages, KV heads, 16, head size] and scales [pages, KV heads, 16], contiguous, on one device: "
                                 f"got {tuple(t.shape)} {t.dtype} on {t.device}")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.n_pages, self.heads, self.head_dim, self.device = shape[0], shape[1], shape[3], k.device
        self.kind = (self.heads, self.head_dim, k.device.index)  # what a context has to have, too
        self._c = lr_fp8_cache(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), shape[0])
        self.c = C.addressof(self._c)
        self.kv = lr_kv_cache(KV_FP8, *(getattr(self._c, n) for n, _ in lr_fp8_cache._fields_))
        self.any, self.raw = C.addressof(self.kv), bytes(self.kv)

    @staticmethod
    def empty(model, n_pages: int, device="cuda:0") -> "Fp8Cache":
        """A cache of zeros (scale bytes 127: 2^0)."""
        shape = (n_pages, int(model.n_kv_heads), 16, int(model.head_dim))
        codes = [torch.zeros(shape, dtype=torch.uint8, device=device).view(torch.float8_e4m3fn) for _ in range(2)]
        return Fp8Cache(*codes, *(torch.full(shape[:3], 127, dtype=torch.uint8, device=device).view(torch.float8_e8m0fnu) for _ in range(2)))


class Fp4Cache:
    """``lr_fp4_cache`` over four tensors of the caller's: code bytes [pages, KV heads, 16, head size / 2] (``torch.uint8``) and scales
    [pages, KV heads, 16, head size / 32] (``torch.float8_e8m0fnu`` or ``torch.uint8``), of K and of V.  ``empty`` makes them."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor):
        shape = k.shape
        for t, want, kinds in ((k, shape, (torch.uint8,)), (v, shape, (torch.uint8,)), (k_scale, shape[:3] + (shape[-1] // 16,), (torch.float8_e8m0fnu, torch.uint8)),
                               (v_scale, shape[:3] + (shape[-1] // 16,), (torch.float8_e8m0fnu, torch.uint8))):
            if t.shape != want or len(shape) != 4 or shape[2] != 16 or shape[3] % 16 != 0 or t.dtype not in kinds or not t.is_contiguous() or t.device != k.device:
                raise ValueError(f"a 4-bit cache is code bytes [pages, KV heads, 16, head size / 2] and scales [pages, KV heads, 16, head size / 32], contiguous, on one device: "
                                 f"got {tuple(t.shape)} {t.dtype} on {t.device}")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.n_pages, self.heads, self.head_dim, self.device = shape[0], shape[1], 2 * shape[3], k.device
        self.kind = (self.heads, self.head_dim, k.device.index)
        self._c = lr_fp4_cache(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), shape[0])
        self.c = C.addressof(self._c)
        self.kv = lr_kv_cache(KV_FP4, *(getattr(self._c, n) for n, _ in lr_fp8_cache._fields_))
        self.any, self.raw = C.addressof(self.kv), bytes(self.kv)

    @staticmethod
    def empty(model, n_pages: int, device="cuda:0") -> "Fp4Cache":
        """A cache of zeros (scale bytes 127: 2^0)."""
        shape = (n_pages, int(model.n_kv_heads), 16, int(model.head_dim))
        codes = [torch.zeros(shape[:3] + (shape[3] // 2,), dtype=torch.uint8, device=device) for _ in range(2)]
        return Fp4Cache(*codes, *(torch.full(shape[:3] + (shape[3] // 32,), 127, dtype=torch.uint8, device=device).view(torch.float8_e8m0fnu) for _ in range(2)))


class Bf16Cache:
    """The bf16 pools [pages, KV heads, 16, head size] of K and of V, as the calls on a cache of any kind take them."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor):
        for t in (k, v):
            if t.shape != k.shape or t.dim() != 4 or t.shape[2] != 16 or t.dtype is not torch.bfloat16 or not t.is_contiguous() or t.device != k.device:
                raise ValueError(f"a bf16 cache is two pools [pages, KV heads, 16, head size], contiguous, on one device: got {tuple(t.shape)} {t.dtype} on {t.device}")
        self.k, self.v = k, v
        self.n_pages, self.heads, self.head_dim, self.device = k.shape[0], k.shape[1], k.shape[3], k.device
        self.kind = (self.heads, self.head_dim, k.device.index)
        self.kv = lr_kv_cache(KV_BF16, k.data_ptr(), v.data_ptr(), None, None, k.shape[0])
        self.any, self.raw = C.addressof(self.kv), bytes(self.kv)


class Rope:
    """``lr_rope``: rotary positions of the first ``rot_dim`` channels of a head.  scaling: "none", "linear", "parts" or "smooth", with its factor and,
    for the latter two, the original length and the turns over it between which frequencies pass from stretched (``lo``) to kept (``hi``)."""

    SCALINGS = ("none", "linear", "parts", "smooth")

    def __init__(self, rot_dim: int, base: float = 10000.0, interleaved: bool = False, scaling: str = "none", factor: float = 1.0, original: float = 0.0,
                 lo: float = 1.0, hi: Optional[float] = None, amplitude: float = 0.0):
        if scaling not in self.SCALINGS:
            raise ValueError(f"scaling is one of {self.SCALINGS}, not {scaling!r}")
        hi = (4.0 if scaling == "smooth" else 32.0) if hi is None else hi
        self.handle = None
        h = C.c_void_p()
        spec = lr_rope_spec(rot_dim, int(interleaved), self.SCALINGS.index(scaling), base, factor, original, lo, hi, amplitude)
        _check(lib().lr_rope_create(C.byref(h), C.byref(spec)), "lr_rope_create")
        self.handle, self.rot_dim = h, rot_dim

    def frequencies(self) -> tuple:
        """(radians a position of every pair, float64 [rot_dim / 2]; amplitude)."""
        f, amplitude = np.empty(self.rot_dim // 2), C.c_double()
        _check(lib().lr_rope_frequencies(self.handle, _addr(f), C.byref(amplitude)), "lr_rope_frequencies")
        return f, amplitude.value

    def close(self):
        if self.handle:
            lib().lr_rope_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _check_cache(cache, ctx: "Context") -> None:
    # what the C side cannot see: how large the tensors behind its pointers are, and where
    if cache.kind != ctx.cache_kind:
        m = ctx.model
        raise ValueError(f"the cache has {cache.heads} heads of {cache.head_dim} on {cache.device}, the context {m.n_kv_heads} of {m.head_dim} on cuda:{ctx.device}")


def _cache_rows(ctx: "Context", cache, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, status: Optional[torch.Tensor]) -> tuple:
    """Number of tokens and the rows' strides, with the tensors found to be what the C side takes them for."""
    _check_cache(cache, ctx)
    n, heads, width, dev = slots.numel(), cache.heads, cache.head_dim, ctx.device
    strides = ()
    if k.shape == v.shape == (n, heads, width) and k.dtype is v.dtype is torch.bfloat16 and k.get_device() == v.get_device() == dev:
        (k_row, k_head, k_one), (v_row, v_head, v_one) = k.stride(), v.stride()
        if n == 0 or (k_one == v_one == 1 and k_head == v_head == width):
            strides = (k_row, v_row) if n > 1 else (heads * width, heads * width)
    if not strides:
        raise ValueError(f"rows are bf16 [{n}, {heads}, {width}] on {cache.device}, a token's heads side by side: got " +
                         " and ".join(f"{tuple(t.shape)} {t.dtype} strides {t.stride()} on {t.device}" for t in (k, v)))
    if slots.dtype is not torch.int64 or not slots.is_contiguous() or slots.get_device() != dev:
        raise ValueError(f"slots are contiguous int64 on {cache.device}")
    if status is not None and (status.dtype is not torch.int32 or status.numel() < 2 or not status.is_contiguous() or status.get_device() != dev):
        raise ValueError(f"status is two int32 on {cache.device}")
    return n, *strides


def _flat(t: Optional[torch.Tensor], kind: torch.dtype, n: int, dev: int) -> bool:
    """Whether the C side may take t for n numbers of that kind side by side (None is its own affair)."""
    return t is None or (t.dtype is kind and t.numel() >= n and t.is_contiguous() and t.get_device() == dev)


def _logit_rows(t: Optional[torch.Tensor], n: int, vocab: int, dev: int) -> bool:
    return t is None or (t.dtype is torch.bfloat16 and t.dim() == 2 and t.shape[0] >= n and t.shape[1] >= vocab and t.stride(1) == 1 and t.get_device() == dev)


def _refuse(where: str, dev: int, **wanted) -> None:
    """The first of the tensors that is not what it has to be: name=(whether it is, the tensor, what it has to be)."""
    for name, (fine, t, want) in wanted.items():
        if not fine:
            raise ValueError(f"{where}: {name} is {want} on device {dev}: got {tuple(t.shape)} {t.dtype} strides {t.stride()} on {t.device}")


def _check_drafted(ctx: "Context", logits, draft_logits, draft_ids, cu_draft, u_accept, u_final, n_accept, final_id, p_draft, q_draft, scratch,
                   scratch_bytes: int) -> tuple:
    """(branches, target rows) of a drafted acceptance, its tensors found to be what the C side takes them for: it sees neither how long they are nor of which kind."""
    dev, vocab, where = ctx.device, ctx.model.vocab, "lr_accept_sample_drafted"
    _refuse(where, dev, cu_draft=(_flat(cu_draft, torch.int32, 1, dev), cu_draft, "int32 [branches + 1]"),
            logits=(_logit_rows(logits, 0, vocab, dev), logits, f"bf16 [rows, >= {vocab}], a row's logits side by side,"))
    n_branch, n_rows = cu_draft.numel() - 1, logits.shape[0]
    n = n_rows - n_branch  # drafts
    if n < 0:
        raise ValueError(f"{where}: {n_branch} branches have a row of logits each at least, not {n_rows} together")
    fine = [_flat(draft_ids, torch.int32, n, dev), _flat(u_accept, torch.float32, n, dev), _flat(u_final, torch.float32, n_branch, dev),
            _flat(n_accept, torch.int32, n_branch, dev), _flat(final_id, torch.int32, n_branch, dev), _flat(p_draft, torch.float32, n, dev),
            _flat(q_draft, torch.float32, n, dev), n == 0 or _logit_rows(draft_logits, n, vocab, dev),
            scratch is None or (scratch.is_contiguous() and scratch.get_device() == dev and scratch.numel() * scratch.element_size() >= scratch_bytes)]
    if not all(fine):
        names = ("draft_ids", "u_accept", "u_final", "n_accept", "final_id", "p_draft", "q_draft", "draft_logits", "scratch")
        tensors = (draft_ids, u_accept, u_final, n_accept, final_id, p_draft, q_draft, draft_logits, scratch)
        want = (f"int32 [{n}]", f"float32 [{n}]", f"float32 [{n_branch}]", f"int32 [{n_branch}]", f"int32 [{n_branch}]", f"float32 [{n}]", f"float32 [{n}]",
                f"bf16 [{n}, >= {vocab}], a row's logits side by side,", f"{scratch_bytes} bytes")
        _refuse(where, dev, **dict(zip(names, zip(fine, tensors, want))))
    return n_branch, n_rows


def _of_kind(cache, kind):
    """The cache, found to be of the kind whose struct the C side will take it for."""
    if not isinstance(cache, kind):
        raise ValueError(f"the call takes a {kind.__name__}, not {type(cache).__name__}")
    return cache


def _check_rope(ctx: "Context", n: int, positions, q, q_out, turned: bool) -> int:
    """The stride of the queries' rows, with the tensors of lr_rope_write found to be what the C side takes them for."""
    m, dev = ctx.model, ctx.device
    heads, width = m.n_q_heads, m.head_dim
    if turned and (positions is None or positions.dtype is not torch.int32 or positions.numel() != n or not positions.is_contiguous() or positions.get_device() != dev):
        raise ValueError(f"lr_rope_write: positions are contiguous int32 [{n}] on device {dev}")
    if q is None or q_out is None:
        if q is not q_out:
            raise ValueError("lr_rope_write: q and q_out come together")
        return 0
    row, head, one = q.stride() if q.dim() == 3 else (0, 0, 0)
    if not (q.shape == (n, heads, width) and q.dtype is torch.bfloat16 and q.get_device() == dev and (n == 0 or (one == 1 and head == width))):
        raise ValueError(f"lr_rope_write: q is bf16 [{n}, {heads}, {width}] on device {dev}, a token's heads side by side: got {tuple(q.shape)} {q.dtype} strides {q.stride()} on {q.device}")
    if not (q_out.dtype is torch.bfloat16 and q_out.is_contiguous() and q_out.get_device() == dev and q_out.numel() == n * heads * width):
        raise ValueError(f"lr_rope_write: q_out is contiguous bf16 [{n}, {heads}, {width}] on device {dev}: got {tuple(q_out.shape)} {q_out.dtype} strides {q_out.stride()} on {q_out.device}")
    return row if n > 1 else heads * width


# (These run before every launch, where each look at a tensor takes a twentieth of a microsecond: all of them in one expression, and who is at fault only then.)
def _check_attention(ctx: "Context", n_q_rows: int, q, out, lse, where: str = "lr_verify_attention_fp8") -> tuple:
    """The addresses of the tensors of an attention call, found to be what the C side takes them for."""
    m, dev = ctx.model, ctx.device
    n = n_q_rows * m.n_q_heads
    if (q is not None and out is not None and lse is not None and q.dtype is out.dtype is torch.bfloat16 and lse.dtype is torch.float32
            and q.get_device() == out.get_device() == lse.get_device() == dev and q.is_contiguous() and out.is_contiguous() and lse.is_contiguous()
            and q.numel() >= n * m.head_dim <= out.numel() and lse.numel() >= n):
        return q.data_ptr(), out.data_ptr(), lse.data_ptr()
    shape = f"[{n_q_rows}, {m.n_q_heads}"
    _refuse(where, dev, q=(_flat(q, torch.bfloat16, n * m.head_dim, dev), q, f"contiguous bf16 {shape}, {m.head_dim}]"),
            out=(_flat(out, torch.bfloat16, n * m.head_dim, dev), out, f"contiguous bf16 {shape}, {m.head_dim}]"),
            lse=(_flat(lse, torch.float32, n, dev), lse, f"contiguous float32 {shape}]"))
    return _ptr(q), _ptr(out), _ptr(lse)


def _check_compact(ctx: "Context", n_req: int, keep_off, keep_pages, keep_valid, new_len, n_pages_kept, where: str = "lr_compact_fp8") -> tuple:
    # (how much of the lists there is to read the offsets say, which are on the device)
    dev, i32 = ctx.device, torch.int32
    some = keep_off is not None and keep_pages is not None and keep_valid is not None and new_len is not None and n_pages_kept is not None
    if (some and keep_off.dtype is keep_pages.dtype is keep_valid.dtype is new_len.dtype is n_pages_kept.dtype is i32
            and keep_off.get_device() == keep_pages.get_device() == keep_valid.get_device() == new_len.get_device() == n_pages_kept.get_device() == dev
            and keep_off.is_contiguous() and keep_pages.is_contiguous() and keep_valid.is_contiguous() and new_len.is_contiguous() and n_pages_kept.is_contiguous()
            and keep_off.numel() > n_req <= new_len.numel() and n_pages_kept.numel() >= n_req and keep_valid.numel() >= keep_pages.numel()):
        return keep_off.data_ptr(), keep_pages.data_ptr(), keep_valid.data_ptr(), new_len.data_ptr(), n_pages_kept.data_ptr()
    _refuse(where, dev, keep_off=(_flat(keep_off, i32, n_req + 1, dev), keep_off, f"int32 [{n_req + 1}]"),
            keep_pages=(_flat(keep_pages, i32, 0, dev), keep_pages, "int32 [page slots]"),
            keep_valid=(_flat(keep_valid, i32, 0 if keep_pages is None else keep_pages.numel(), dev), keep_valid, "int32, as long as keep_pages,"),
            new_len=(_flat(new_len, i32, n_req, dev), new_len, f"int32 [{n_req}]"), n_pages_kept=(_flat(n_pages_kept, i32, n_req, dev), n_pages_kept, f"int32 [{n_req}]"))
    return _ptr(keep_off), _ptr(keep_pages), _ptr(keep_valid), _ptr(new_len), _ptr(n_pages_kept)


class Context:
    """``lr_ctx``: one per (device, model geometry)."""

    def __init__(self, model, device: int = 0):
        self.model = model
        self.device = device
        self.cache_kind = (int(model.n_kv_heads), int(model.head_dim), device)
        h = C.c_void_p()
        m = _model_struct(model)
        _check(lib().lr_create(C.byref(h), C.byref(m), device), "lr_create")
        self.handle = h
        # Handles of the plans that are left: plans are destroyed before their context, also where the collector finalises both in
        # whatever order (weak references to them are dead by then).
        self._open = set()

    def close(self):
        if self.handle:
            while self._open:
                lib().lr_plan_destroy(self._open.pop())
            lib().lr_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def launch_count(self) -> int:
        return int(lib().lr_launch_count(self.handle))

    def lr_accept_greedy(self, logits: torch.Tensor, draft_ids: torch.Tensor, cu_draft: torch.Tensor, n_accept: torch.Tensor,
                         bonus_id: torch.Tensor, scratch: torch.Tensor, row_argmax: Optional[torch.Tensor] = None,
                         stream=None) -> None:
        """logits [n_rows, >=vocab] bf16 (row stride = logits.stride(0)); outputs int32 [n_branch]."""
        n_branch = cu_draft.numel() - 1
        n_rows = logits.shape[0]
        _check(lib().lr_accept_greedy(self.handle, _ptr(logits), logits.stride(0), _ptr(draft_ids), _ptr(cu_draft), n_branch,
                                      n_rows, _ptr(n_accept), _ptr(bonus_id), _ptr(row_argmax), _ptr(scratch),
                                      _stream_ptr(stream)), "lr_accept_greedy")

    def lr_accept_greedy_static(self, logits: torch.Tensor, draft_ids: torch.Tensor, cu_draft: torch.Tensor,
                                n_accept: torch.Tensor, bonus_id: torch.Tensor, row_argmax: Optional[torch.Tensor] = None,
                                stream=None) -> None:
        """``lr_accept_greedy`` on the scratch array built into the library: no scratch argument and no
        device allocation; at most ``ACCEPT_STATIC_MAX_ROWS`` logits rows."""
        n_branch = cu_draft.numel() - 1
        _check(lib().lr_accept_greedy_static(self.handle, _ptr(logits), logits.stride(0), _ptr(draft_ids), _ptr(cu_draft),
                                             n_branch, logits.shape[0], _ptr(n_accept), _ptr(bonus_id), _ptr(row_argmax),
                                             _stream_ptr(stream)), "lr_accept_greedy_static")

    def lr_accept_sample(self, logits: torch.Tensor, draft_ids: torch.Tensor, cu_draft: torch.Tensor, temperature: float,
                         u_accept: torch.Tensor, u_final: torch.Tensor, n_accept: torch.Tensor, final_id: torch.Tensor,
                         scratch: torch.Tensor, p_draft: Optional[torch.Tensor] = None, stream=None) -> None:
        """Rejection-sampling acceptance; u_accept [sum L] and u_final [n_branch] are fp32 uniforms in [0, 1)."""
        n_branch = cu_draft.numel() - 1
        _check(lib().lr_accept_sample(self.handle, _ptr(logits), logits.stride(0), _ptr(draft_ids), _ptr(cu_draft), n_branch,
                                      logits.shape[0], float(temperature), _ptr(u_accept), _ptr(u_final), _ptr(n_accept),
                                      _ptr(final_id), _ptr(p_draft), _ptr(scratch), _stream_ptr(stream)), "lr_accept_sample")

    def lr_accept_sample_filtered(self, logits: torch.Tensor, draft_ids: torch.Tensor, cu_draft: torch.Tensor,
                                  temperature: float, top_k: int, top_p: float, u_accept: torch.Tensor, u_final: torch.Tensor,
                                  n_accept: torch.Tensor, final_id: torch.Tensor, scratch: torch.Tensor,
                                  p_draft: Optional[torch.Tensor] = None, n_kept: Optional[torch.Tensor] = None,
                                  stream=None) -> None:
        """``lr_accept_sample`` on the target distribution after the top-k / top-p filters (0 and 1.0 switch them off)."""
        n_branch = cu_draft.numel() - 1
        _check(lib().lr_accept_sample_filtered(self.handle, _ptr(logits), logits.stride(0), _ptr(draft_ids), _ptr(cu_draft),
                                               n_branch, logits.shape[0], float(temperature), int(top_k), float(top_p),
                                               _ptr(u_accept), _ptr(u_final), _ptr(n_accept), _ptr(final_id), _ptr(p_draft),
                                               _ptr(n_kept), _ptr(scratch), _stream_ptr(stream)), "lr_accept_sample_filtered")

    def lr_accept_sample_drafted(self, logits: torch.Tensor, draft_logits: torch.Tensor, draft_ids: torch.Tensor, cu_draft: torch.Tensor,
                                 temperature: float, draft_temperature: float, u_accept: torch.Tensor, u_final: torch.Tensor, n_accept: torch.Tensor,
                                 final_id: torch.Tensor, scratch: torch.Tensor, p_draft: Optional[torch.Tensor] = None,
                                 q_draft: Optional[torch.Tensor] = None, stream=None) -> None:
        """Rejection-sampling acceptance of drafts that a draft model sampled; draft_logits [sum L, >= vocab] are what they were drawn from."""
        n_branch, n_rows = _check_drafted(self, logits, draft_logits, draft_ids, cu_draft, u_accept, u_final, n_accept, final_id, p_draft, q_draft, scratch,
                                          self._drafted_scratch_bytes(logits.shape[0]))
        _check(lib().lr_accept_sample_drafted(self.handle, _ptr(logits), logits.stride(0), _ptr(draft_logits), draft_logits.stride(0), _ptr(draft_ids),
                                              _ptr(cu_draft), n_branch, n_rows, temperature, draft_temperature, _ptr(u_accept), _ptr(u_final),
                                              _ptr(n_accept), _ptr(final_id), _ptr(p_draft), _ptr(q_draft), _ptr(scratch),
                                              _stream_on(self.device, stream)), "lr_accept_sample_drafted")

    def _drafted_scratch_bytes(self, n_rows: int) -> int:
        n = C.c_size_t()
        _check(lib().lr_accept_sample_drafted_scratch_bytes(self.handle, n_rows, C.byref(n)), "lr_accept_sample_drafted_scratch_bytes")
        return n.value

    def accept_sample_drafted_scratch(self, n_rows: int) -> torch.Tensor:
        return torch.empty((self._drafted_scratch_bytes(n_rows) + 7) // 8, dtype=torch.int64, device=f"cuda:{self.device}")

    def lr_fp8_write(self, cache: Fp8Cache, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, status: Optional[torch.Tensor] = None,
                     stream=None) -> None:
        """Quantises rows [tokens, KV heads, head size] (bf16; a slice of a joint projection's output will do) into the cache's token
        slots (int64: page * 16 + place, negative: none); status: two int32 of zeros that a slot beyond the cache sets."""
        n, k_stride, v_stride = _cache_rows(self, _of_kind(cache, Fp8Cache), k, v, slots, status)
        _check(lib().lr_fp8_write(self.handle, cache.c, k.data_ptr(), k_stride, v.data_ptr(), v_stride, slots.data_ptr(), n, _ptr(status),
                                  _stream_on(self.device, stream)), "lr_fp8_write")

    def lr_fp8_read(self, cache: Fp8Cache, slots: torch.Tensor, k: torch.Tensor, v: torch.Tensor, status: Optional[torch.Tensor] = None,
                    stream=None) -> None:
        """The values at the token slots, into rows as ``lr_fp8_write`` takes them; a row without a slot is left as it was."""
        n, k_stride, v_stride = _cache_rows(self, _of_kind(cache, Fp8Cache), k, v, slots, status)
        _check(lib().lr_fp8_read(self.handle, cache.c, slots.data_ptr(), n, k.data_ptr(), k_stride, v.data_ptr(), v_stride, _ptr(status),
                                 _stream_on(self.device, stream)), "lr_fp8_read")

    def lr_fp4_write(self, cache: Fp4Cache, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, status: Optional[torch.Tensor] = None,
                     stream=None) -> None:
        """``lr_fp8_write`` into a 4-bit cache."""
        n, k_stride, v_stride = _cache_rows(self, _of_kind(cache, Fp4Cache), k, v, slots, status)
        _check(lib().lr_fp4_write(self.handle, cache.c, k.data_ptr(), k_stride, v.data_ptr(), v_stride, slots.data_ptr(), n, _ptr(status),
                                  _stream_on(self.device, stream)), "lr_fp4_write")

    def lr_fp4_read(self, cache: Fp4Cache, slots: torch.Tensor, k: torch.Tensor, v: torch.Tensor, status: Optional[torch.Tensor] = None,
                    stream=None) -> None:
        """``lr_fp8_read`` from a 4-bit cache."""
        n, k_stride, v_stride = _cache_rows(self, _of_kind(cache, Fp4Cache), k, v, slots, status)
        _check(lib().lr_fp4_read(self.handle, cache.c, slots.data_ptr(), n, k.data_ptr(), k_stride, v.data_ptr(), v_stride, _ptr(status),
                                 _stream_on(self.device, stream)), "lr_fp4_read")

    def lr_rope_write(self, rope: Optional[Rope], positions: Optional[torch.Tensor], cache, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor,
                      q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None, stream=None) -> None:
        """Turns the queries q [tokens, q heads, head size] into q_out and the keys k into the cache's slots, V beside them: rows of a joint projection, as
        ``lr_fp8_write`` takes them.  positions: int32 [tokens].  cache: a ``Bf16Cache``, ``Fp8Cache`` or ``Fp4Cache``.  Without rope nothing is turned."""
        n, k_stride, v_stride = _cache_rows(self, cache, k, v, slots, status)
        if rope is not None and rope.handle is None:
            raise ValueError("lr_rope_write: the rope is closed")
        q_stride = _check_rope(self, n, positions, q, q_out, rope is not None)
        _check(lib().lr_rope_write(self.handle, None if rope is None else rope.handle, cache.any, _ptr(positions), _ptr(q), q_stride, _ptr(q_out),
                                   k.data_ptr(), k_stride, v.data_ptr(), v_stride, slots.data_ptr(), n, _ptr(status), _stream_on(self.device, stream)),
               "lr_rope_write")

    def lr_copy_pages(self, src, dst, src_pages: torch.Tensor, dst_pages: torch.Tensor, status: Optional[torch.Tensor] = None, stream=None) -> None:
        """Copies pages src_pages[i] of every cache of ``src`` to dst_pages[i] of its counterpart in ``dst`` (a cache or a list of them, a layer each)."""
        if isinstance(src, (list, tuple)):
            if not isinstance(dst, (list, tuple)) or len(src) != len(dst):
                raise ValueError(f"lr_copy_pages: {len(src)} caches to copy from, and others to copy to")
            for c in (*src, *dst):
                _check_cache(c, self)
            n_caches, src_at, dst_at = len(src), b"".join([c.raw for c in src]), b"".join([c.raw for c in dst])
        else:
            if isinstance(dst, (list, tuple)):
                raise ValueError(f"lr_copy_pages: one cache to copy from, {len(dst)} to copy to")
            _check_cache(src, self)
            _check_cache(dst, self)
            n_caches, src_at, dst_at = 1, src.any, dst.any
        dev, i32 = self.device, torch.int32
        n = src_pages.numel()
        if not (src_pages.dtype is dst_pages.dtype is i32 and dst_pages.numel() == n and src_pages.get_device() == dst_pages.get_device() == dev
                and src_pages.is_contiguous() and dst_pages.is_contiguous() and (status is None or _flat(status, i32, 2, dev))):
            _refuse("lr_copy_pages", dev, src_pages=(_flat(src_pages, i32, n, dev), src_pages, f"int32 [{n}]"),
                    dst_pages=(_flat(dst_pages, i32, n, dev) and dst_pages.numel() == n, dst_pages, f"int32 [{n}]"),
                    status=(_flat(status, i32, 2, dev), status, "two int32"))
        _check(lib().lr_copy_pages(self.handle, src_at, dst_at, n_caches, src_pages.data_ptr(), dst_pages.data_ptr(), n, _ptr(status), _stream_on(dev, stream)),
               "lr_copy_pages")

    def accept_sample_filtered_scratch(self, n_rows: int) -> torch.Tensor:
        n = C.c_size_t()
        _check(lib().lr_accept_sample_filtered_scratch_bytes(self.handle, n_rows, C.byref(n)),
               "lr_accept_sample_filtered_scratch_bytes")
        return torch.empty((n.value + 7) // 8, dtype=torch.int64, device=f"cuda:{self.device}")

    def accept_sample_scratch(self, n_rows: int) -> torch.Tensor:
        n = C.c_size_t()
        _check(lib().lr_accept_sample_scratch_bytes(self.handle, n_rows, C.byref(n)), "lr_accept_sample_scratch_bytes")
        return torch.empty((n.value + 7) // 8, dtype=torch.int64, device=f"cuda:{self.device}")

    @staticmethod
    def accept_scratch(n_rows: int, device) -> torch.Tensor:
        n = C.c_size_t()
        _check(lib().lr_accept_scratch_bytes(n_rows, C.byref(n)), "lr_accept_scratch_bytes")
        return torch.zeros((n.value + 7) // 8, dtype=torch.int64, device=device)


class Plan:
    """``lr_plan``: device tables and the attention work partition of one batch."""

    def __init__(self, ctx: Context, batch, stream=None):
        self.ctx = ctx
        self.host = HostBatch(batch)
        n, draft, h = C.c_size_t(), C.c_void_p(), C.c_void_p()
        _check(lib().lr_plan_begin(ctx.handle, C.byref(self.host.c), C.byref(n), C.byref(draft)), "lr_plan_begin")
        try:
            self.workspace_bytes = n.value
            self.workspace = torch.empty(n.value + 256, dtype=torch.uint8, device=ctx.device)
            start = self.workspace.data_ptr()
            self._ws_ptr = start + (-start) % 256
            stream = _stream_ptr(stream)
        except BaseException:
            lib().lr_plan_drop(draft)
            raise
        _check(lib().lr_plan_finish(draft, self._ws_ptr, n.value, stream, C.byref(h)), "lr_plan_finish")
        self.handle, self._open = h, ctx._open
        self._open.add(h.value)
        self.n_req = self.host.c.n_req
        self.n_branch = self.host.c.n_branch
        self.n_page_slots = self.host.c.n_page_slots
        self.n_q_rows = int(batch.cu_q[-1])

    def close(self):
        if self.handle:
            if self.handle.value in self._open:  # else its context has destroyed it
                self._open.remove(self.handle.value)
                lib().lr_plan_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def lr_plan_set_attention_path(self, path: int) -> None:
        _check(lib().lr_plan_set_attention_path(self.handle, path), "lr_plan_set_attention_path")

    def lr_plan_debug_set_page(self, page_slot: int, new_id: int, stream=None) -> None:
        _check(lib().lr_plan_debug_set_page(self.handle, page_slot, new_id, _stream_ptr(stream)), "lr_plan_debug_set_page")

    def lr_plan_debug_set_wait_limit(self, microseconds: int) -> None:
        _check(lib().lr_plan_debug_set_wait_limit(self.handle, microseconds), "lr_plan_debug_set_wait_limit")

    def lr_plan_debug_set_phantom_bytes(self, n_bytes: int) -> None:
        _check(lib().lr_plan_debug_set_phantom_bytes(self.handle, n_bytes), "lr_plan_debug_set_phantom_bytes")

    def lr_plan_describe(self) -> dict:
        info = lr_plan_info()
        _check(lib().lr_plan_describe(self.handle, C.byref(info)), "lr_plan_describe")
        return {n: int(getattr(info, n)) for n, _ in lr_plan_info._fields_}

    def lr_verify_attention(self, q, k_pool, v_pool, out, lse=None, softmax_scale: float = 0.0, stream=None) -> None:
        _check(lib().lr_verify_attention(self.handle, _ptr(q), _ptr(k_pool), _ptr(v_pool), _ptr(out), _ptr(lse),
                                         float(softmax_scale), _stream_ptr(stream)), "lr_verify_attention")

    def lr_commit(self, verdict, n_accept, n_steps_accepted, survivor, committed_len, keep_off, keep_pages, keep_valid,
                  free_off, free_pages, stream=None) -> None:
        _check(lib().lr_commit(self.handle, _ptr(verdict), _ptr(n_accept), _ptr(n_steps_accepted), _ptr(survivor),
                               _ptr(committed_len), _ptr(keep_off), _ptr(keep_pages), _ptr(keep_valid), _ptr(free_off),
                               _ptr(free_pages), _stream_ptr(stream)), "lr_commit")

    def compact_scratch(self) -> torch.Tensor:
        n = C.c_size_t()
        _check(lib().lr_compact_scratch_bytes(self.handle, C.byref(n)), "lr_compact_scratch_bytes")
        t = torch.empty(n.value + 256, dtype=torch.uint8, device=f"cuda:{self.ctx.device}")
        off = (-t.data_ptr()) % 256
        return t[off : off + n.value]

    def lr_compact(self, keep_off, keep_pages, keep_valid, k_pool, v_pool, new_len, n_pages_kept, scratch, stream=None) -> None:
        """Moves the committed tokens (keep lists of ``lr_commit``) densely into the leading kept pages, in place."""
        _check(lib().lr_compact(self.handle, _ptr(keep_off), _ptr(keep_pages), _ptr(keep_valid), _ptr(k_pool), _ptr(v_pool),
                                _ptr(new_len), _ptr(n_pages_kept), _ptr(scratch), _stream_ptr(stream)), "lr_compact")

    def lr_verify_attention_fp8(self, q, cache: Fp8Cache, out, lse=None, softmax_scale: float = 0.0, stream=None) -> None:
        """``lr_verify_attention`` over an 8-bit cache."""
        _check_cache(_of_kind(cache, Fp8Cache), self.ctx)
        q_at, out_at, lse_at = _check_attention(self.ctx, self.n_q_rows, q, out, lse)
        _check(lib().lr_verify_attention_fp8(self.handle, q_at, cache.c, out_at, lse_at, float(softmax_scale), _stream_on(self.ctx.device, stream)),
               "lr_verify_attention_fp8")

    def lr_compact_fp8(self, keep_off, keep_pages, keep_valid, cache: Fp8Cache, new_len, n_pages_kept, stream=None) -> None:
        """``lr_compact`` over an 8-bit cache: codes and scales together."""
        _check_cache(_of_kind(cache, Fp8Cache), self.ctx)
        off_at, pages_at, valid_at, len_at, kept_at = _check_compact(self.ctx, self.n_req, keep_off, keep_pages, keep_valid, new_len, n_pages_kept)
        _check(lib().lr_compact_fp8(self.handle, off_at, pages_at, valid_at, cache.c, len_at, kept_at, _stream_on(self.ctx.device, stream)),
               "lr_compact_fp8")

    def lr_verify_attention_fp4(self, q, cache: Fp4Cache, out, lse=None, softmax_scale: float = 0.0, stream=None) -> None:
        """``lr_verify_attention`` over a 4-bit cache."""
        _check_cache(_of_kind(cache, Fp4Cache), self.ctx)
        q_at, out_at, lse_at = _check_attention(self.ctx, self.n_q_rows, q, out, lse, "lr_verify_attention_fp4")
        _check(lib().lr_verify_attention_fp4(self.handle, q_at, cache.c, out_at, lse_at, float(softmax_scale), _stream_on(self.ctx.device, stream)),
               "lr_verify_attention_fp4")

    def lr_compact_fp4(self, keep_off, keep_pages, keep_valid, cache: Fp4Cache, new_len, n_pages_kept, stream=None) -> None:
        """``lr_compact`` over a 4-bit cache: codes and scales together."""
        _check_cache(_of_kind(cache, Fp4Cache), self.ctx)
        off_at, pages_at, valid_at, len_at, kept_at = _check_compact(self.ctx, self.n_req, keep_off, keep_pages, keep_valid, new_len, n_pages_kept, "lr_compact_fp4")
        _check(lib().lr_compact_fp4(self.handle, off_at, pages_at, valid_at, cache.c, len_at, kept_at, _stream_on(self.ctx.device, stream)),
               "lr_compact_fp4")

    def lr_poll_status(self, stream=None) -> int:
        d = C.c_int32()
        _check(lib().lr_poll_status(self.handle, _stream_ptr(stream), C.byref(d)), "lr_poll_status")
        return d.value

    def pass_staging(self) -> torch.Tensor:
        n = C.c_size_t()
        _check(lib().lr_pass_staging_bytes(self.handle, C.byref(n)), "lr_pass_staging_bytes")
        t = torch.zeros(n.value + 256, dtype=torch.uint8, device=f"cuda:{self.ctx.device}")
        return t

    def lr_verify_pass(self, ctx: Context, q, k_pool, v_pool, out, lse, logits, draft_ids, cu_draft, n_accept, bonus_id, row_argmax, accept_scratch,
                       verdict, n_steps_accepted, survivor, committed_len, keep_off, keep_pages, keep_valid, free_off, free_pages,
                       softmax_scale: float = 0.0, side=None, stream=None) -> None:
        """Attention, greedy acceptance and commit in one call; ``side`` is a stream for the latter two."""
        io = _PASS_IO(q.data_ptr(), k_pool.data_ptr(), v_pool.data_ptr(), out.data_ptr(), 0 if lse is None else lse.data_ptr(),
                      logits.data_ptr(), draft_ids.data_ptr(), cu_draft.data_ptr(), n_accept.data_ptr(), bonus_id.data_ptr(),
                      0 if row_argmax is None else row_argmax.data_ptr(), accept_scratch.data_ptr(), verdict.data_ptr(),
                      n_steps_accepted.data_ptr(), survivor.data_ptr(), committed_len.data_ptr(), keep_off.data_ptr(),
                      keep_pages.data_ptr(), keep_valid.data_ptr(), free_off.data_ptr(), free_pages.data_ptr(), logits.stride(0),
                      logits.shape[0])
        _check(lib().lr_verify_pass(ctx.handle, self.handle, io, softmax_scale, 0 if side is None else side.cuda_stream, _stream_ptr(stream)),
               "lr_verify_pass")

    def lr_verify_pass_host(self, io: lr_pass_host_io, k_pool, v_pool, staging: torch.Tensor, softmax_scale: float = 0.0,
                            stream=None) -> None:
        off = (-staging.data_ptr()) % 256
        _check(lib().lr_verify_pass_host(self.handle, C.byref(io), _ptr(k_pool), _ptr(v_pool), staging.data_ptr() + off,
                                         staging.numel() - off, float(softmax_scale), _stream_ptr(stream)),
               "lr_verify_pass_host")


# ---- host-side cycle model (no device needed) --------------------------------------------------------
def _stats(st: lr_cycle_stats) -> dict:
    return {n: int(getattr(st, n)) for n, _ in lr_cycle_stats._fields_}


def lr_cycle_simulate_sync(gamma: int, num: int, den: int, verdicts) -> dict:
    v = np.ascontiguousarray(verdicts, dtype=np.uint8)
    st = lr_cycle_stats()
    _check(lib().lr_cycle_simulate_sync(gamma, num, den, v.ctypes.data, len(v), C.byref(st)), "lr_cycle_simulate_sync")
    return _stats(st)


def lr_cycle_simulate_async(gamma: int, num: int, den: int, verdicts) -> dict:
    v = np.ascontiguousarray(verdicts, dtype=np.uint8)
    st = lr_cycle_stats()
    _check(lib().lr_cycle_simulate_async(gamma, num, den, v.ctypes.data, len(v), C.byref(st)), "lr_cycle_simulate_async")
    return _stats(st)


def lr_cycle_speedup(mode: int, k: int, alpha: float, c: float) -> float:
    return float(lib().lr_cycle_speedup(mode, k, alpha, c))


def lr_cycle_best_strategy(budget: int, alpha1: float, c1: float, alpha2: float, c2: float, asynchronous: bool = True):
    k1, k2, h = C.c_int32(), C.c_int32(), C.c_double()
    _check(lib().lr_cycle_best_strategy(budget, alpha1, c1, alpha2, c2, int(asynchronous), C.byref(k1), C.byref(k2),
                                        C.byref(h)), "lr_cycle_best_strategy")
    return k1.value, k2.value, h.value
