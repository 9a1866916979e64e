"""Thin ctypes binding of libapm.so: same names as the C ABI, argument marshalling only.

Every step of the path runs in the library's HIP kernels; nothing here computes.  The library must
have been built (python -m paper_2303_02868_amd.build); loading fails loudly otherwise.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from typing import Optional, Sequence

_PKG = os.path.dirname(os.path.abspath(__file__))
# APM_LIBRARY selects another build of the same library (e.g. one compiled with different tunables).
LIB_PATH = os.environ.get("APM_LIBRARY") or os.path.join(_PKG, "libapm.so")

APM_OK, APM_EINVAL, APM_ENOMEM, APM_ERANGE, APM_EDEVICE, APM_ESTATE = 0, -1, -2, -3, -4, -5
APM_DEV_GPU, APM_DEV_HOST, APM_DEV_FILE = 0, 1, 2
APM_F32, APM_BF16 = 0, 1
APM_P32, APM_M32, APM_V32, APM_G16, APM_P16, APM_N_STATES = 0, 1, 2, 3, 4, 5
APM_SKIP_NONE, APM_SKIP_UNTOUCHED = 0, 1
APM_POOL_NO_ZERO = 1
APM_POOL_FILE_DIRECT = 2
APM_STREAM_STAGED, APM_STREAM_DIRECT, APM_STREAM_STAGED_DMA = 0, 1, 2
APM_K_REDUCE, APM_K_UPDATE, APM_K_SEGCOPY, APM_N_KERNEL_CLASSES = 0, 1, 2, 3
APM_CKPT_I8, APM_CKPT_F8, APM_CKPT_BLOCK = 0, 1, 32
APM_NORM_NONE, APM_NORM_RMS, APM_NORM_LAYER = 0, 1, 2
APM_GATE_NONE, APM_GATE_CHANNEL, APM_GATE_TOKEN, APM_GATE_FULL = 0, 1, 2, 3
APM_JOIN_MAX_COLS = 16384
ALL_STATES = 0b11111
FP32_STATES = 0b00111
B16_STATES = 0b11000

EXPORTS = [
    "apm_last_error", "apm_pack_plan", "apm_pool_create", "apm_pool_destroy",
    "apm_pool_pages_in_use", "apm_pool_page_info", "apm_pool_state_ptr", "apm_pool_set_layout",
    "apm_pack_tensors", "apm_unpack", "apm_page_adamw_step", "apm_page_adamw_step_fused",
    "apm_page_copy_async",
    "apm_schedule_plan", "apm_file_pool_create", "apm_tiered_create", "apm_tiered_destroy", "apm_tiered_io_bytes", "apm_tiered_set_range", "apm_streamer_set_page_count", "apm_tiered_step", "apm_tiered_step_delayed", "apm_streamer_step_scheduled", "apm_streamer_step_delayed", "apm_streamer_create", "apm_streamer_destroy", "apm_streamer_step", "apm_streamer_copy_only", "apm_streamer_set_cache", "apm_cache_pages_that_fit", "apm_streamer_set_host_first_page", "apm_streamer_set_mode", "apm_streamer_get_mode", "apm_streamer_probe_rates", "apm_step_delayed",
    "apm_delayed_applied", "apm_delayed_set_outputs", "apm_delayed_grad_buffer", "apm_delayed_accumulate", "apm_pool_set_timing", "apm_pool_read_timing",
    "apm_page_adamw_step_noalloc", "apm_noalloc_scratch_bytes", "apm_noalloc_max_pages",
    "apm_streamer_overlap_report",
    "apm_streamer_set_host_write_through",
    "apm_ckpt_write", "apm_ckpt_read", "apm_norm_join_forward", "apm_norm_join_backward",
    "apm_norm_join_workspace_bytes", "apm_ckpt_weight_grad", "apm_ckpt_weight_grad_workspace_bytes",
]


class apm_pool_desc(C.Structure):
    _fields_ = [("device", C.c_int32), ("hip_device", C.c_int32), ("page_elems", C.c_int64),
                ("n_pages", C.c_int64), ("state_mask", C.c_uint32), ("flags", C.c_uint32),
                ("base", C.c_void_p * APM_N_STATES)]


class apm_tensor(C.Structure):
    _fields_ = [("id", C.c_int64), ("dtype", C.c_int32), ("reserved", C.c_int32),
                ("numel", C.c_int64), ("data", C.c_void_p)]


class apm_segment(C.Structure):
    _fields_ = [("tensor", C.c_int64), ("tensor_off", C.c_int64), ("page", C.c_int64),
                ("page_off", C.c_int64), ("n", C.c_int64)]

    def astuple(self):
        return (self.tensor, self.tensor_off, self.page, self.page_off, self.n)


class apm_page_info(C.Structure):
    _fields_ = [("total_elems", C.c_int64), ("used_elems", C.c_int64),
                ("available_elems", C.c_int64), ("device", C.c_int32), ("n_tensors", C.c_int32),
                ("tensor_id", C.c_int64 * 2), ("tensor_elems", C.c_int64 * 2)]


class apm_task(C.Structure):
    _fields_ = [("op", C.c_int32), ("trigger_id", C.c_int32), ("target", C.c_int64)]


APM_TASK_MOVE_TO_GPU, APM_TASK_COMPUTE = 0, 1


class apm_hyper(C.Structure):
    _fields_ = [("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double),
                ("eps", C.c_double), ("weight_decay", C.c_double), ("max_grad_norm", C.c_double),
                ("skip_mode", C.c_int32), ("reserved", C.c_int32)]


class apm_matrix(C.Structure):
    _fields_ = [("data", C.c_void_p), ("stride", C.c_int64), ("dtype", C.c_int32), ("reserved", C.c_int32)]


class apm_vector(C.Structure):
    _fields_ = [("data", C.c_void_p), ("dtype", C.c_int32), ("reserved", C.c_int32)]


class apm_ckpt(C.Structure):
    _fields_ = [("q", C.c_void_p), ("scale", C.c_void_p), ("q_stride", C.c_int64), ("scale_stride", C.c_int64),
                ("format", C.c_int32), ("reserved", C.c_int32)]


class apm_norm(C.Structure):
    _fields_ = [("kind", C.c_int32), ("reserved", C.c_int32), ("eps", C.c_double), ("weight", apm_vector),
                ("bias", apm_vector), ("ckpt", apm_ckpt), ("rstd", C.c_void_p)]


class apm_norm_join(C.Structure):
    _fields_ = [("rows", C.c_int64), ("cols", C.c_int64), ("residual_scale", C.c_double), ("x", apm_matrix),
                ("branch", apm_matrix), ("y", apm_matrix), ("n", apm_matrix), ("gate", apm_matrix),
                ("gate_kind", C.c_int32), ("reserved", C.c_int32), ("pre", apm_norm), ("post", apm_norm)]


class apm_norm_join_grads(C.Structure):
    _fields_ = [("dn", apm_matrix), ("dy", apm_matrix), ("dx", apm_matrix), ("dbranch", apm_matrix),
                ("dgate", apm_matrix), ("dpre_weight", apm_vector), ("dpre_bias", apm_vector),
                ("dpost_weight", apm_vector), ("dpost_bias", apm_vector)]


class apm_weight_grad(C.Structure):
    _fields_ = [("tokens", C.c_int64), ("out", C.c_int64), ("in", C.c_int64), ("n_groups", C.c_int64),
                ("offsets", C.c_void_p), ("dy", apm_matrix), ("kept", apm_ckpt), ("weight", apm_vector),
                ("bias", apm_vector), ("dw", apm_matrix), ("dw_group_stride", C.c_int64), ("db", apm_vector),
                ("accumulate", C.c_int32), ("reserved", C.c_int32)]


class ApmError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"apm error {code}: {msg}")
        self.code = code


_lib = None


def lib() -> C.CDLL:
    """The loaded library.  Raises if it has not been built: there is no fallback path."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2303_02868_amd.build`")
    L = C.CDLL(LIB_PATH)
    vp, i64, i32 = C.c_void_p, C.c_int64, C.c_int
    P = C.POINTER
    L.apm_last_error.restype = C.c_char_p
    L.apm_last_error.argtypes = []
    L.apm_pack_plan.argtypes = [i64, P(i64), i64, P(apm_segment), P(i64), P(i64), P(C.c_double)]
    L.apm_pool_create.argtypes = [P(vp), P(apm_pool_desc)]
    L.apm_pool_destroy.argtypes = [vp]
    L.apm_pool_pages_in_use.argtypes = [vp]
    L.apm_pool_pages_in_use.restype = i64
    L.apm_pool_page_info.argtypes = [vp, i64, P(apm_page_info)]
    L.apm_pool_state_ptr.argtypes = [vp, i32, i64]
    L.apm_pool_state_ptr.restype = vp
    L.apm_pool_set_layout.argtypes = [vp, P(apm_tensor), i64, P(apm_segment), P(i64), P(i64),
                                      P(C.c_double), vp]
    L.apm_pack_tensors.argtypes = [vp, i32, P(apm_tensor), i64, P(apm_segment), P(i64), P(i64),
                                   P(C.c_double), vp]
    L.apm_unpack.argtypes = [vp, i32, P(apm_tensor), i64, vp]
    L.apm_page_adamw_step.argtypes = [vp, P(i64), i64, i64, P(apm_hyper), vp, vp, vp]
    L.apm_page_adamw_step_fused.argtypes = [vp, P(i64), i64, i64, P(apm_hyper), P(apm_tensor),
                                            P(apm_tensor), i64, vp, vp, vp]
    L.apm_page_copy_async.argtypes = [vp, i64, vp, i64, i64, i32, vp]
    L.apm_page_adamw_step_noalloc.argtypes = [vp, i64, i64, P(apm_hyper), vp, vp, vp]
    L.apm_noalloc_scratch_bytes.argtypes = []
    L.apm_noalloc_scratch_bytes.restype = C.c_size_t
    L.apm_noalloc_max_pages.argtypes = [i64]
    L.apm_noalloc_max_pages.restype = i64
    L.apm_schedule_plan.argtypes = [P(i64), P(i64), P(i64), i64, P(i64), i64, i64, i64, P(apm_task), P(i64), P(i64)]
    L.apm_streamer_step_scheduled.argtypes = [vp, P(apm_task), i64, P(i64), i64, P(i64), i64, P(apm_hyper), vp, vp, vp]
    L.apm_streamer_step_delayed.argtypes = [vp, vp, P(apm_hyper), vp]
    L.apm_file_pool_create.argtypes = [P(vp), C.c_char_p, i32, i64, i64, C.c_uint32, C.c_uint32]
    L.apm_tiered_create.argtypes = [P(vp), vp, vp, i64, i32, i32]
    L.apm_tiered_destroy.argtypes = [vp]
    L.apm_tiered_step.argtypes = [vp, i64, P(apm_hyper), vp, vp, vp]
    L.apm_tiered_io_bytes.argtypes = [vp, P(i64), P(i64)]
    L.apm_tiered_set_range.argtypes = [vp, i64, i64]
    L.apm_streamer_set_page_count.argtypes = [vp, i64]
    L.apm_tiered_step_delayed.argtypes = [vp, vp, P(apm_hyper), vp]
    L.apm_streamer_create.argtypes = [P(vp), vp, vp, i64, i32]
    L.apm_streamer_destroy.argtypes = [vp]
    L.apm_streamer_step.argtypes = [vp, i64, P(apm_hyper), vp, vp, vp]
    L.apm_streamer_copy_only.argtypes = [vp, i32, vp]
    L.apm_streamer_set_cache.argtypes = [vp, vp, i64]
    L.apm_streamer_set_host_first_page.argtypes = [vp, i64]
    L.apm_cache_pages_that_fit.argtypes = [i32, i64, i64, C.c_size_t, P(i64)]
    L.apm_streamer_set_mode.argtypes = [vp, i32, i32, i32]
    L.apm_streamer_get_mode.argtypes = [vp]
    L.apm_streamer_probe_rates.argtypes = [vp, P(C.c_double), P(C.c_double), P(C.c_double)]
    L.apm_streamer_overlap_report.argtypes = [vp, P(C.c_int), P(C.c_int)]
    L.apm_streamer_set_host_write_through.argtypes = [vp, C.c_int]
    L.apm_step_delayed.argtypes = [vp, P(i64), i64, vp, P(apm_hyper), vp]
    L.apm_delayed_accumulate.argtypes = [vp, P(i64), i64, vp, vp]
    L.apm_delayed_grad_buffer.argtypes = [vp, vp]
    L.apm_delayed_grad_buffer.restype = vp
    L.apm_delayed_applied.argtypes = [vp]
    L.apm_delayed_applied.restype = i64
    L.apm_delayed_set_outputs.argtypes = [vp, vp, vp]
    L.apm_pool_set_timing.argtypes = [vp, i32]
    L.apm_pool_read_timing.argtypes = [vp, P(C.c_double), P(i64)]
    L.apm_ckpt_write.argtypes = [i64, i64, P(apm_matrix), P(apm_ckpt), vp]
    L.apm_ckpt_read.argtypes = [i64, i64, P(apm_ckpt), P(apm_matrix), vp]
    L.apm_norm_join_forward.argtypes = [P(apm_norm_join), vp]
    L.apm_norm_join_backward.argtypes = [P(apm_norm_join), P(apm_norm_join_grads), vp, C.c_size_t, vp]
    L.apm_norm_join_workspace_bytes.argtypes = [i64, i64]
    L.apm_norm_join_workspace_bytes.restype = C.c_size_t
    L.apm_ckpt_weight_grad.argtypes = [P(apm_weight_grad), vp, C.c_size_t, vp]
    L.apm_ckpt_weight_grad_workspace_bytes.argtypes = [P(apm_weight_grad)]
    L.apm_ckpt_weight_grad_workspace_bytes.restype = C.c_size_t
    for name in EXPORTS:
        getattr(L, name)              # every declared entry point must be exported
    _lib = L
    return L


def apm_last_error() -> str:
    return lib().apm_last_error().decode()


def _check(rc: int) -> None:
    if rc != APM_OK:
        raise ApmError(rc, apm_last_error())


def _ptr(x) -> Optional[int]:
    """Raw address of a torch tensor / numpy array / int / None."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    if hasattr(x, "data_ptr"):
        return x.data_ptr()
    if hasattr(x, "ctypes"):
        return x.ctypes.data
    raise TypeError(type(x))


def _stream(stream) -> Optional[int]:
    if stream is None:
        return None
    if isinstance(stream, int):
        return stream or None
    return stream.cuda_stream or None          # torch.cuda.Stream


def _i64_array(xs: Optional[Sequence[int]]):
    if xs is None:
        return None, 0
    arr = (C.c_int64 * len(xs))(*[int(x) for x in xs])
    return arr, len(xs)


def make_hyper(lr=1e-4, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, max_grad_norm=0.0,
               skip_mode=APM_SKIP_NONE) -> apm_hyper:
    return apm_hyper(lr, beta1, beta2, eps, weight_decay, max_grad_norm, skip_mode, 0)


def make_tensors(numels: Sequence[int], dtype: int, datas: Optional[Sequence] = None,
                 ids: Optional[Sequence[int]] = None):
    n = len(numels)
    arr = (apm_tensor * max(n, 1))()
    for i in range(n):
        arr[i].id = i if ids is None else int(ids[i])
        arr[i].dtype = dtype
        arr[i].numel = int(numels[i])
        arr[i].data = None if datas is None else _ptr(datas[i])
    return arr


class PlanResult:
    """segs: a list of (tensor, tensor_off, page, page_off, n), or the library's array of `n_segs` of them, which becomes
    that list when it is first looked at: tuples for every segment cost a pack of small tensors several times its kernel
    (5.4 M bf16 elements in 64 K pages, us a call: 35.9 with the list, 7.7 without)."""

    def __init__(self, segs, n_pages, fragmentation, n_segs=None):
        if n_segs is None:
            self.segments = segs
        else:
            self._segs, self._n = segs, n_segs
        self.n_pages = n_pages
        self.fragmentation = fragmentation

    def __getattr__(self, name):          # `segments` that nobody has looked at yet
        if name != "segments" or "_segs" not in self.__dict__:
            raise AttributeError(name)
        # the array stays: another thread may be at it, and the first of them to end gives the list to all
        return self.__dict__.setdefault("segments", [self._segs[i].astuple() for i in range(self._n)])


def apm_pack_plan(page_elems: int, numels: Sequence[int]) -> PlanResult:
    L = lib()
    arr, n = _i64_array(numels)
    n_segs, n_pages, frag = C.c_int64(0), C.c_int64(0), C.c_double(0)
    _check(L.apm_pack_plan(page_elems, arr, n, None, C.byref(n_segs), C.byref(n_pages), C.byref(frag)))
    segs = (apm_segment * max(1, n_segs.value))()
    cap = C.c_int64(n_segs.value)
    _check(L.apm_pack_plan(page_elems, arr, n, segs, C.byref(cap), C.byref(n_pages), C.byref(frag)))
    return PlanResult(segs, n_pages.value, frag.value, cap.value)


class Pool:
    """Owner of an apm_pool handle."""

    def __init__(self, handle: int, desc: apm_pool_desc, keepalive=None):
        self.handle = handle
        self.desc = desc
        self._keepalive = keepalive

    def destroy(self):
        if self.handle:
            h, self.handle = self.handle, None
            _check(lib().apm_pool_destroy(h))

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def apm_pool_create(device: int, page_elems: int, n_pages: int, state_mask: int = ALL_STATES,
                    flags: int = 0, hip_device: int = 0, base: Optional[dict] = None) -> Pool:
    """base: {state: torch tensor | address} of caller-owned regions (kept alive by the Pool)."""
    d = apm_pool_desc()
    d.device, d.hip_device, d.page_elems, d.n_pages = device, hip_device, page_elems, n_pages
    d.state_mask, d.flags = state_mask, flags
    for s in range(APM_N_STATES):
        d.base[s] = _ptr(base.get(s)) if base else None
    out = C.c_void_p()
    _check(lib().apm_pool_create(C.byref(out), C.byref(d)))
    return Pool(out.value, d, keepalive=base)


def apm_pool_destroy(pool: Pool) -> None:
    pool.destroy()


def apm_pool_pages_in_use(pool: Pool) -> int:
    return lib().apm_pool_pages_in_use(pool.handle)


def apm_pool_page_info(pool: Pool, page: int) -> apm_page_info:
    info = apm_page_info()
    _check(lib().apm_pool_page_info(pool.handle, page, C.byref(info)))
    return info


def apm_pool_state_ptr(pool: Pool, state: int, page: int = 0) -> Optional[int]:
    return lib().apm_pool_state_ptr(pool.handle, state, page)


def apm_pool_set_layout(pool: Pool, tensors, n: int, stream=None) -> PlanResult:
    L = lib()
    cap = 2 * pool.desc.n_pages + 2
    segs = (apm_segment * cap)()
    n_segs, n_pages, frag = C.c_int64(cap), C.c_int64(0), C.c_double(0)
    _check(L.apm_pool_set_layout(pool.handle, tensors, n, segs, C.byref(n_segs), C.byref(n_pages),
                                 C.byref(frag), _stream(stream)))
    return PlanResult(segs, n_pages.value, frag.value, n_segs.value)


def apm_pack_tensors(pool: Pool, state: int, tensors, n: int, stream=None) -> PlanResult:
    L = lib()
    cap = 2 * pool.desc.n_pages + 2
    segs = (apm_segment * cap)()
    n_segs, n_pages, frag = C.c_int64(cap), C.c_int64(0), C.c_double(0)
    _check(L.apm_pack_tensors(pool.handle, state, tensors, n, segs, C.byref(n_segs),
                              C.byref(n_pages), C.byref(frag), _stream(stream)))
    return PlanResult(segs, n_pages.value, frag.value, n_segs.value)


def apm_unpack(pool: Pool, state: int, tensors, n: int, stream=None) -> None:
    _check(lib().apm_unpack(pool.handle, state, tensors, n, _stream(stream)))


def apm_page_adamw_step(pool: Pool, pages: Optional[Sequence[int]], n_pages: int, step: int,
                        hyper: apm_hyper, grad_norm=None, skip_mask=None, stream=None) -> None:
    arr, _ = _i64_array(pages)
    _check(lib().apm_page_adamw_step(pool.handle, arr, n_pages, step, C.byref(hyper),
                                     _ptr(grad_norm), _ptr(skip_mask), _stream(stream)))


def apm_page_adamw_step_fused(pool: Pool, pages: Optional[Sequence[int]], n_pages: int, step: int,
                              hyper: apm_hyper, grad_tensors, p16_tensors, n_tensors: int,
                              grad_norm=None, skip_mask=None, stream=None) -> None:
    arr, _ = _i64_array(pages)
    _check(lib().apm_page_adamw_step_fused(pool.handle, arr, n_pages, step, C.byref(hyper),
                                           grad_tensors, p16_tensors, n_tensors, _ptr(grad_norm),
                                           _ptr(skip_mask), _stream(stream)))


def apm_page_adamw_step_noalloc(pool: Pool, n_pages: int, step: int, hyper: apm_hyper,
                                grad_norm=None, skip_mask=None, stream=None) -> None:
    _check(lib().apm_page_adamw_step_noalloc(pool.handle, n_pages, step, C.byref(hyper),
                                             _ptr(grad_norm), _ptr(skip_mask), _stream(stream)))


def apm_noalloc_scratch_bytes() -> int:
    return lib().apm_noalloc_scratch_bytes()


def apm_noalloc_max_pages(page_elems: int) -> int:
    return lib().apm_noalloc_max_pages(page_elems)


def apm_page_copy_async(dst: Pool, dst_page: int, src: Pool, src_page: int, n_pages: int,
                        state: int, stream=None) -> None:
    _check(lib().apm_page_copy_async(dst.handle, dst_page, src.handle, src_page, n_pages, state,
                                     _stream(stream)))


def apm_file_pool_create(path_prefix: str, page_elems: int, n_pages: int, state_mask: int = FP32_STATES,
                         flags: int = 0, hip_device: int = 0) -> Pool:
    d = apm_pool_desc()
    d.device, d.hip_device, d.page_elems, d.n_pages = APM_DEV_FILE, hip_device, page_elems, n_pages
    d.state_mask, d.flags = state_mask, flags
    out = C.c_void_p()
    _check(lib().apm_file_pool_create(C.byref(out), path_prefix.encode(), hip_device, page_elems, n_pages,
                                      state_mask, flags))
    return Pool(out.value, d)


class Tiered:
    def __init__(self, handle, file: Pool, dev: Pool):
        self.handle, self.file, self.dev = handle, file, dev

    def destroy(self):
        if self.handle:
            h, self.handle = self.handle, None
            _check(lib().apm_tiered_destroy(h))

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def apm_tiered_create(file: Pool, dev: Pool, batch_pages: int, n_slots: int, io_threads: int) -> Tiered:
    out = C.c_void_p()
    _check(lib().apm_tiered_create(C.byref(out), file.handle, dev.handle, batch_pages, n_slots, io_threads))
    return Tiered(out.value, file, dev)


def apm_tiered_destroy(t: Tiered) -> None:
    t.destroy()


def apm_tiered_set_range(t: Tiered, first_page: int, n_pages: int = -1) -> None:
    _check(lib().apm_tiered_set_range(t.handle, first_page, n_pages))


def apm_streamer_set_page_count(s: "Streamer", n_pages: int) -> None:
    _check(lib().apm_streamer_set_page_count(s.handle, n_pages))


def apm_tiered_io_bytes(t: Tiered):
    """(bytes read, bytes written) queued since creation."""
    r, w = C.c_int64(0), C.c_int64(0)
    _check(lib().apm_tiered_io_bytes(t.handle, C.byref(r), C.byref(w)))
    return r.value, w.value


def apm_tiered_step(t: Tiered, step: int, hyper: apm_hyper, grad_norm=None, skip_mask=None, stream=None) -> None:
    _check(lib().apm_tiered_step(t.handle, step, C.byref(hyper), _ptr(grad_norm), _ptr(skip_mask), _stream(stream)))


def apm_tiered_step_delayed(t: Tiered, new_g16, hyper: apm_hyper, stream=None) -> None:
    _check(lib().apm_tiered_step_delayed(t.handle, _ptr(new_g16), C.byref(hyper), _stream(stream)))


class Streamer:
    def __init__(self, handle, host: Pool, dev: Pool):
        self.handle, self.host, self.dev = handle, host, dev

    def destroy(self):
        if self.handle:
            h, self.handle = self.handle, None
            _check(lib().apm_streamer_destroy(h))

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def apm_schedule_plan(layers: Sequence, last_access: Optional[Sequence[int]], page_bytes: int,
                      gpu_memory_bytes: int):
    """layers: sequence of (page_list, bytes).  Returns ([(op, target, trigger_id), ...], peak_bytes)."""
    offsets, pages, sizes = [0], [], []
    for page_list, nbytes in layers:
        pages.extend(int(p) for p in page_list)
        offsets.append(len(pages))
        sizes.append(int(nbytes))
    off_a, _ = _i64_array(offsets)
    pg_a, n_pages = _i64_array(pages)
    sz_a, n_layers = _i64_array(sizes)
    la_a = _i64_array(last_access)[0] if last_access is not None else None
    cap = n_pages + n_layers
    tasks = (apm_task * max(1, cap))()
    n_tasks, peak = C.c_int64(cap), C.c_int64(0)
    _check(lib().apm_schedule_plan(off_a, pg_a, sz_a, n_layers, la_a, n_pages, page_bytes, gpu_memory_bytes,
                                   tasks, C.byref(n_tasks), C.byref(peak)))
    return [(tasks[i].op, tasks[i].target, tasks[i].trigger_id) for i in range(n_tasks.value)], peak.value


def apm_streamer_create(host: Pool, dev: Pool, batch_pages: int, n_slots: int) -> Streamer:
    out = C.c_void_p()
    _check(lib().apm_streamer_create(C.byref(out), host.handle, dev.handle, batch_pages, n_slots))
    return Streamer(out.value, host, dev)


def apm_streamer_destroy(s: Streamer) -> None:
    s.destroy()


def apm_streamer_step(s: Streamer, step: int, hyper: apm_hyper, grad_norm=None, skip_mask=None,
                      stream=None) -> None:
    _check(lib().apm_streamer_step(s.handle, step, C.byref(hyper), _ptr(grad_norm),
                                   _ptr(skip_mask), _stream(stream)))


def apm_streamer_step_scheduled(s: Streamer, tasks: Sequence, layer_first_page: Sequence[int], step: int,
                                hyper: apm_hyper, grad_norm=None, skip_mask=None, stream=None,
                                last_access: Optional[Sequence[int]] = None) -> None:
    """tasks: [(op, target, trigger_id), ...] as apm_schedule_plan returns them."""
    arr = (apm_task * max(1, len(tasks)))()
    for i, (op, target, trig) in enumerate(tasks):
        arr[i].op, arr[i].target, arr[i].trigger_id = op, target, trig
    lf, n1 = _i64_array(layer_first_page)
    la = _i64_array(last_access)[0] if last_access is not None else None
    _check(lib().apm_streamer_step_scheduled(s.handle, arr, len(tasks), lf, n1 - 1, la, step, C.byref(hyper),
                                             _ptr(grad_norm), _ptr(skip_mask), _stream(stream)))


def apm_streamer_set_host_write_through(s: Streamer, on: bool) -> None:
    _check(lib().apm_streamer_set_host_write_through(s.handle, int(bool(on))))


def apm_streamer_overlap_report(s: Streamer):
    """(update stream, pipeline streams): 1 runs beside the producer stream, 0 does not, -1 not measured."""
    a, b = C.c_int(-1), C.c_int(-1)
    _check(lib().apm_streamer_overlap_report(s.handle, C.byref(a), C.byref(b)))
    return a.value, b.value


def apm_streamer_step_delayed(s: Streamer, new_g16, hyper: apm_hyper, stream=None) -> None:
    _check(lib().apm_streamer_step_delayed(s.handle, _ptr(new_g16), C.byref(hyper), _stream(stream)))


def apm_streamer_set_cache(s: Streamer, cache: Optional[Pool], n_resident: int) -> None:
    _check(lib().apm_streamer_set_cache(s.handle, cache.handle if cache else None, n_resident))
    s.cache = cache


def apm_cache_pages_that_fit(page_elems: int, n_pages: int, reserve_bytes: int = 0, hip_device: int = 0) -> int:
    out = C.c_int64(0)
    _check(lib().apm_cache_pages_that_fit(hip_device, page_elems, n_pages, reserve_bytes, C.byref(out)))
    return out.value


def apm_streamer_set_host_first_page(s: Streamer, first_model_page: int) -> None:
    _check(lib().apm_streamer_set_host_first_page(s.handle, first_model_page))


def apm_streamer_set_mode(s: Streamer, mode: int, direct_wavefronts: int = 0,
                          wavefronts_per_workgroup: int = 0) -> None:
    _check(lib().apm_streamer_set_mode(s.handle, mode, direct_wavefronts, wavefronts_per_workgroup))


def apm_streamer_get_mode(s: Streamer) -> int:
    m = lib().apm_streamer_get_mode(s.handle)
    _check(min(m, 0))
    return m


def apm_streamer_probe_rates(s: Streamer):
    """(copy-in alone, copy-out alone, each way when both run) in GB/s, from creation."""
    a, b, c = C.c_double(), C.c_double(), C.c_double()
    _check(lib().apm_streamer_probe_rates(s.handle, C.byref(a), C.byref(b), C.byref(c)))
    return a.value, b.value, c.value


def apm_streamer_copy_only(s: Streamer, directions: int, stream=None) -> None:
    _check(lib().apm_streamer_copy_only(s.handle, directions, _stream(stream)))


def apm_step_delayed(pool: Pool, pages: Optional[Sequence[int]], n_pages: int, new_g16,
                     hyper: apm_hyper, stream=None) -> None:
    arr, _ = _i64_array(pages)
    _check(lib().apm_step_delayed(pool.handle, arr, n_pages, _ptr(new_g16), C.byref(hyper),
                                  _stream(stream)))


def apm_delayed_accumulate(pool: Pool, pages: Optional[Sequence[int]], n_pages: int, g16, stream=None) -> None:
    arr, _ = _i64_array(pages)
    _check(lib().apm_delayed_accumulate(pool.handle, arr, n_pages, _ptr(g16), _stream(stream)))


def apm_delayed_grad_buffer(pool: Pool, stream=None) -> int:
    p = lib().apm_delayed_grad_buffer(pool.handle, _stream(stream))
    if not p:
        raise ApmError(APM_EDEVICE, apm_last_error())
    return p


def apm_delayed_applied(pool: Pool) -> int:
    return lib().apm_delayed_applied(pool.handle)


def apm_delayed_set_outputs(pool: Pool, grad_norm=None, skip_mask=None) -> None:
    _check(lib().apm_delayed_set_outputs(pool.handle, _ptr(grad_norm), _ptr(skip_mask)))


def apm_pool_set_timing(pool: Pool, enable: bool) -> None:
    _check(lib().apm_pool_set_timing(pool.handle, int(enable)))


def apm_pool_read_timing(pool: Pool):
    """({class: total ms}, {class: launches}) since the last read."""
    ms = (C.c_double * APM_N_KERNEL_CLASSES)()
    n = (C.c_int64 * APM_N_KERNEL_CLASSES)()
    _check(lib().apm_pool_read_timing(pool.handle, ms, n))
    return list(ms), list(n)


# ---- activations --------------------------------------------------------------------------------
# Tensors in, raw structures out: these look at shapes, strides, types and memory (that of the current device, on which the calls'
# kernels run), which the structures do not all carry.  The large structures are packed in one go: field by field they cost more than
# the smallest calls' kernels (a join of eight tokens, us of host time: 33 field by field, 19 packed).  As everywhere here, stream=None is
# the null stream and not torch's current one: inside torch.cuda.stream(s), or in a capture, pass stream=s.

_DTYPES: dict = {}
_NO_MATRIX, _NO_VECTOR, _NO_CKPT = (0, 0, 0, 0), (0, 0, 0), (0, 0, 0, 0, 0, 0)
_MATRIX, _VECTOR, _CKPT = "Qqii", "Qii", "QQqqii"
_NORM = "iid" + _VECTOR * 2 + _CKPT + "Q"
_pack_join = struct.Struct("<qqd" + _MATRIX * 5 + "ii" + _NORM * 2).pack
_pack_grads = struct.Struct("<" + _MATRIX * 5 + _VECTOR * 4).pack
_pack_weight_grad = struct.Struct("<qqqqQ" + _MATRIX + _CKPT + _VECTOR * 2 + _MATRIX + "q" + _VECTOR + "ii").pack


def _dtype(t) -> int:
    code = _DTYPES.get(t.dtype)
    if code is None:
        code = {"torch.float32": APM_F32, "torch.bfloat16": APM_BF16}.get(str(t.dtype))
        if code is None:
            raise ValueError(f"a tensor of {t.dtype}: float32 or bfloat16 is needed")
        _DTYPES[t.dtype] = code
    return code


_current_device = None


def _here():
    """The current device, on which a call's kernels run; None where the process has one GPU and nothing to tell apart (looking costs the smallest
    calls 0.5 to 1 us of 6 to 16), -2 where none is in use."""
    return _first_here() if _current_device is None else _current_device()


def _first_here():
    global _current_device
    import torch
    if not torch.cuda.is_initialized():
        return -2
    _current_device = torch.cuda.current_device if torch.cuda.device_count() > 1 else lambda: None
    return _current_device()


def _elsewhere(name, t, here) -> int:
    device = t.get_device()                # -1: host memory
    if device >= 0:                        # with several GPUs in use
        raise ValueError(f"{name} is on GPU {device}, the current one is {here}")
    if not t.is_pinned():
        raise ValueError(f"{name} is in memory that the GPU cannot address")
    return t.data_ptr()


def _same_gpu(made, here) -> None:
    if made != here and made is not None:  # None: a structure that its owner filled by hand
        raise ValueError(f"the tensors were looked at for GPU {made}, the current one is {here}")


def _matrix(name, t, rows, cols, here):
    if t is None:
        return _NO_MATRIX
    stride, code = t.stride(), _DTYPES.get(t.dtype)
    if t.shape != (rows, cols) or (stride[1] != 1 and cols > 1):
        raise ValueError(f"{name}: {tuple(t.shape)} with strides {stride}, {rows} rows of {cols} contiguous elements are needed")
    at = t.data_ptr() if (t.is_cuda if here is None else t.get_device() == here) else _elsewhere(name, t, here)
    return at, stride[0], _dtype(t) if code is None else code, 0


def _vector(name, t, n, here):
    if t is None:
        return _NO_VECTOR
    if t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name}: {tuple(t.shape)} with strides {t.stride()}, {n} contiguous elements are needed")
    code = _DTYPES.get(t.dtype)
    at = t.data_ptr() if (t.is_cuda if here is None else t.get_device() == here) else _elsewhere(name, t, here)
    return at, _dtype(t) if code is None else code, 0


def make_matrix(name: str, t, rows: int, cols: int) -> apm_matrix:
    """The apm_matrix of a two-dimensional tensor (None: not given) that has to be rows x cols."""
    return apm_matrix(*_matrix(name, t, rows, cols, _here()))


def make_vector(name: str, t, n: int) -> apm_vector:
    return apm_vector(*_vector(name, t, n, _here()))


class Ckpt:
    """An 8-bit matrix: the tensors, and the words of its apm_ckpt."""
    __slots__ = ("shape", "words", "tensors", "device")


def make_ckpt(q, scale, format: int) -> Ckpt:
    """q: rows x cols of one byte each (any type), scale: rows x ceil(cols / 32) likewise."""
    c = Ckpt()
    rows, cols = c.shape = q.shape
    nb = -(-cols // APM_CKPT_BLOCK)
    q_stride, s_stride = q.stride(), scale.stride()
    if q.element_size() != 1 or scale.element_size() != 1 or scale.shape != (rows, nb) or (q_stride[1] != 1 and cols > 1) or (s_stride[1] != 1 and nb > 1):
        raise ValueError(f"an 8-bit matrix of {tuple(q.shape)} needs bytes, and scales of {(rows, nb)}: got {tuple(scale.shape)}")
    here = c.device = _here()
    c.words = (q.data_ptr() if (q.is_cuda if here is None else q.get_device() == here) else _elsewhere("q", q, here),
               scale.data_ptr() if (scale.is_cuda if here is None else scale.get_device() == here) else _elsewhere("scale", scale, here),
               q_stride[0], s_stride[0], format, 0)
    c.tensors = q, scale
    return c


def _ckpt_words(name, c, rows, cols, here):
    if c is None:
        return _NO_CKPT
    if c.shape != (rows, cols):
        raise ValueError(f"{name}: {tuple(c.shape)}, {(rows, cols)} is needed")
    if c.device != here:
        _same_gpu(c.device, here)
    return c.words


def apm_ckpt_write(x, ckpt: Ckpt, stream=None) -> None:
    (rows, cols), here = ckpt.shape, _here()
    _check(lib().apm_ckpt_write(rows, cols, apm_matrix(*_matrix("x", x, rows, cols, here)), apm_ckpt(*_ckpt_words("ckpt", ckpt, rows, cols, here)),
                                _stream(stream)))


def apm_ckpt_read(ckpt: Ckpt, x, stream=None) -> None:
    (rows, cols), here = ckpt.shape, _here()
    _check(lib().apm_ckpt_read(rows, cols, apm_ckpt(*_ckpt_words("ckpt", ckpt, rows, cols, here)), apm_matrix(*_matrix("x", x, rows, cols, here)),
                               _stream(stream)))


def _gate_shape(kind, rows, cols):
    return (1, cols) if kind == APM_GATE_CHANNEL else (rows, 1) if kind == APM_GATE_TOKEN else (rows, cols)


def _rstd(name, t, rows, here):
    data, dtype, _ = _vector(name, t, rows, here)
    if t is not None and dtype != APM_F32:
        raise ValueError(f"{name} must be float32")
    return data


def make_norm_join(rows: int, cols: int, *, x=None, branch=None, y=None, n=None, residual_scale=1.0, gate_kind=APM_GATE_NONE, gate=None,
                   pre_norm=APM_NORM_NONE, pre_eps=0.0, pre_weight=None, pre_bias=None, pre_ckpt=None, pre_rstd=None,
                   post_norm=APM_NORM_NONE, post_eps=0.0, post_weight=None, post_bias=None, post_ckpt=None, post_rstd=None) -> apm_norm_join:
    """What apm_norm_join_forward and _backward work on.  The tensors are kept alive by it."""
    here = _here()
    j = apm_norm_join.from_buffer_copy(_pack_join(
        rows, cols, residual_scale, *_matrix("x", x, rows, cols, here), *_matrix("branch", branch, rows, cols, here),
        *_matrix("y", y, rows, cols, here), *_matrix("n", n, rows, cols, here), *_matrix("gate", gate, *_gate_shape(gate_kind, rows, cols), here), gate_kind, 0,
        pre_norm, 0, pre_eps, *_vector("pre_weight", pre_weight, cols, here), *_vector("pre_bias", pre_bias, cols, here),
        *_ckpt_words("pre_ckpt", pre_ckpt, rows, cols, here), _rstd("pre_rstd", pre_rstd, rows, here),
        post_norm, 0, post_eps, *_vector("post_weight", post_weight, cols, here), *_vector("post_bias", post_bias, cols, here),
        *_ckpt_words("post_ckpt", post_ckpt, rows, cols, here), _rstd("post_rstd", post_rstd, rows, here)))
    j.shape, j.kind, j.device = (rows, cols), gate_kind, here
    j.tensors = (x, branch, y, n, gate, pre_weight, pre_bias, pre_ckpt, pre_rstd, post_weight, post_bias, post_ckpt, post_rstd)
    return j


def make_norm_join_grads(join: apm_norm_join, *, dn=None, dy=None, dx=None, dbranch=None, dgate=None, dpre_weight=None, dpre_bias=None,
                         dpost_weight=None, dpost_bias=None) -> apm_norm_join_grads:
    """dgate has the gate's shape."""
    (rows, cols), here = join.shape, _here()
    _same_gpu(join.device, here)
    g = apm_norm_join_grads.from_buffer_copy(_pack_grads(
        *_matrix("dn", dn, rows, cols, here), *_matrix("dy", dy, rows, cols, here), *_matrix("dx", dx, rows, cols, here),
        *_matrix("dbranch", dbranch, rows, cols, here), *_matrix("dgate", dgate, *_gate_shape(join.kind, rows, cols), here),
        *_vector("dpre_weight", dpre_weight, cols, here), *_vector("dpre_bias", dpre_bias, cols, here),
        *_vector("dpost_weight", dpost_weight, cols, here), *_vector("dpost_bias", dpost_bias, cols, here)))
    g.tensors = (dn, dy, dx, dbranch, dgate, dpre_weight, dpre_bias, dpost_weight, dpost_bias)
    g.device = here
    return g


def apm_norm_join_forward(join: apm_norm_join, stream=None) -> None:
    _same_gpu(getattr(join, "device", None), _here())
    _check(lib().apm_norm_join_forward(join, _stream(stream)))


def apm_norm_join_workspace_bytes(rows: int, cols: int) -> int:
    return lib().apm_norm_join_workspace_bytes(rows, cols)


def _room(workspace, here):
    if workspace is None:
        return None, 0
    if not workspace.is_contiguous():      # its size would not be what lies behind its address
        raise ValueError(f"workspace: {tuple(workspace.shape)} with strides {workspace.stride()}, contiguous memory is needed")
    at = workspace.data_ptr() if (workspace.is_cuda if here is None else workspace.get_device() == here) else _elsewhere("workspace", workspace, here)
    return at, workspace.numel() * workspace.element_size()


def apm_norm_join_backward(join: apm_norm_join, grads: apm_norm_join_grads, workspace, stream=None) -> None:
    here = _here()
    _same_gpu(getattr(grads, "device", None), here)
    _check(lib().apm_norm_join_backward(join, grads, *_room(workspace, here), _stream(stream)))


def make_weight_grad(dy, kept: Ckpt, dw, *, db=None, weight=None, bias=None, offsets=None, accumulate=False) -> apm_weight_grad:
    """dw: [out, in], or with offsets (int64, groups + 1) [groups, out, in]; db: [out] or [groups, out]."""
    (tokens, k), here = kept.shape, _here()
    out, groups, at = dy.shape[1], 0, 0
    if offsets is not None:
        groups = offsets.numel() - 1
        at = offsets.data_ptr() if (offsets.is_cuda if here is None else offsets.get_device() == here) else _elsewhere("offsets", offsets, here)
        if str(offsets.dtype) != "torch.int64" or not offsets.is_contiguous() or groups < 1 or dw.dim() != 3 or dw.shape[0] != groups:
            raise ValueError(f"offsets {offsets.dtype} of {tuple(offsets.shape)} for gradients of {tuple(dw.shape)}")
    w = apm_weight_grad.from_buffer_copy(_pack_weight_grad(
        tokens, out, k, groups, at, *_matrix("dy", dy, tokens, out, here), *_ckpt_words("kept", kept, tokens, k, here),
        *_vector("weight", weight, k, here), *_vector("bias", bias, k, here), *_matrix("dw", dw[0] if groups else dw, out, k, here),
        dw.stride(0) if groups else 0, *_vector("db", db, max(1, groups) * out, here), int(accumulate), 0))
    w.tensors = (dy, kept, dw, db, weight, bias, offsets)
    w.device = here
    return w


def apm_ckpt_weight_grad_workspace_bytes(grad: apm_weight_grad) -> int:
    return lib().apm_ckpt_weight_grad_workspace_bytes(grad)


def apm_ckpt_weight_grad(grad: apm_weight_grad, workspace=None, stream=None) -> None:
    here = _here()
    _same_gpu(getattr(grad, "device", None), here)
    _check(lib().apm_ckpt_weight_grad(grad, *_room(workspace, here), _stream(stream)))
