"""ctypes binding of libsfb's C-ABI (include/sfb.h).

Argument marshalling only: torch tensors supply device memory and the stream;
every step of the path runs in the library's kernels.  There is no fallback:
if the shared library is missing, importing this module's functions raises.
"""
from __future__ import annotations

import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsfb.so")

SFB_MLR, SFB_DML, SFB_SC = 0, 1, 2
SFB_F32, SFB_BF16 = 0, 1
SFB_PROX_PROJECT, SFB_PROX_NORMALIZE = 0, 1
SFB_OK, SFB_EINVAL, SFB_ENOWS, SFB_EHIP, SFB_ETOOBIG = 0, -1, -2, -3, -4
SFB_STATIC_SCRATCH_BYTES = 32 << 20


class sfb_batch(ctypes.Structure):
    _fields_ = [
        ("X", ctypes.c_void_p),
        ("Y", ctypes.c_void_p),
        ("sim", ctypes.c_void_p),
        ("B", ctypes.c_int64),
        ("in_dtype", ctypes.c_int32),
        ("sf_dtype", ctypes.c_int32),
        ("lambda_", ctypes.c_float),
        ("ista_iters", ctypes.c_int32),
        ("power_iters", ctypes.c_int32),
        ("margin", ctypes.c_float),
    ]


class sfb_csr(ctypes.Structure):
    _fields_ = [
        ("indptr", ctypes.c_void_p),
        ("indices", ctypes.c_void_p),
        ("values", ctypes.c_void_p),
        ("rows", ctypes.c_int64),
        ("cols", ctypes.c_int64),
        ("nnz", ctypes.c_int64),
        ("dtype", ctypes.c_int32),
    ]


class sfb_adapters(ctypes.Structure):
    _fields_ = [
        ("U", ctypes.c_void_p),
        ("V", ctypes.c_void_p),
        ("ranks", ctypes.c_void_p),
        ("scale", ctypes.c_void_p),
        ("count", ctypes.c_int64),
        ("rank", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
    ]


class sfb_requests(ctypes.Structure):
    _fields_ = [("start", ctypes.c_void_p), ("adapter", ctypes.c_void_p), ("count", ctypes.c_int64)]


class sfb_tensor(ctypes.Structure):
    _fields_ = [("src", ctypes.c_void_p), ("dst", ctypes.c_void_p), ("n", ctypes.c_int64), ("dtype", ctypes.c_int32)]


class sfb_kernel_time(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char_p), ("launches", ctypes.c_int32), ("total_ms", ctypes.c_float)]


class SfbError(RuntimeError):
    def __init__(self, code, what, hip=0):
        self.code = code
        self.hip = hip
        super().__init__("%s failed: %d (%s)%s" % (what, code, strerror(code), " hip=%d" % hip if hip else ""))


_lib = None


def lib():
    """The loaded C library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                "libsfb.so is not built (%s); run __graft_entry__.build() or "
                "python paper_1409_5705_amd/build.py" % LIB_PATH)
        L = ctypes.CDLL(LIB_PATH)
        vp, i64, i32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32
        L.sfb_create.argtypes = [ctypes.POINTER(vp), ctypes.c_int, vp]
        L.sfb_create.restype = ctypes.c_int
        L.sfb_destroy.argtypes = [vp]
        L.sfb_destroy.restype = ctypes.c_int
        L.sfb_workspace_bytes.argtypes = [i32, i64, i64, ctypes.POINTER(sfb_batch)]
        L.sfb_workspace_bytes.restype = i64
        L.sfb_apply_workspace_bytes.argtypes = [i64, i64, i64, i32]
        L.sfb_apply_workspace_bytes.restype = i64
        L.sfb_shadow_bytes.argtypes = [i64, i64]
        L.sfb_shadow_bytes.restype = i64
        L.sfb_shadow_attach.argtypes = [vp, vp, i64, i64, vp, i64]
        L.sfb_shadow_attach.restype = ctypes.c_int
        L.sfb_shadow_detach.argtypes = [vp]
        L.sfb_shadow_detach.restype = ctypes.c_int
        L.sfb_split_bytes.argtypes = [i64, i64]
        L.sfb_split_bytes.restype = i64
        L.sfb_split_attach.argtypes = [vp, vp, i64, i64, vp, i64]
        L.sfb_split_attach.restype = ctypes.c_int
        L.sfb_split_export.argtypes = [vp, vp]
        L.sfb_split_export.restype = ctypes.c_int
        L.sfb_split_detach.argtypes = [vp]
        L.sfb_split_detach.restype = ctypes.c_int
        L.sfb_set_workspace.argtypes = [vp, vp, i64]
        L.sfb_set_workspace.restype = ctypes.c_int
        L.sfb_compute_sf.argtypes = [vp, i32, vp, i64, i64, ctypes.POINTER(sfb_batch), vp, vp, vp]
        L.sfb_compute_sf.restype = ctypes.c_int
        L.sfb_apply.argtypes = [vp, vp, i64, i64, vp, vp, i64, i32, ctypes.c_float]
        L.sfb_apply.restype = ctypes.c_int
        L.sfb_apply_static.argtypes = [vp, vp, i64, i64, vp, vp, i64, i32, ctypes.c_float]
        L.sfb_apply_static.restype = ctypes.c_int
        L.sfb_apply_signed_workspace_bytes.argtypes = [i64, i64, i64, i32]
        L.sfb_apply_signed_workspace_bytes.restype = i64
        L.sfb_apply_signed.argtypes = [vp, vp, i64, i64, vp, vp, vp, i64, i32, ctypes.c_float]
        L.sfb_apply_signed.restype = ctypes.c_int
        L.sfb_csr_check.argtypes = [vp, ctypes.POINTER(sfb_csr), ctypes.POINTER(i64)]
        L.sfb_csr_check.restype = ctypes.c_int
        L.sfb_mlr_sf_csr_workspace_bytes.argtypes = [i64, i64, i64, i32]
        L.sfb_mlr_sf_csr_workspace_bytes.restype = i64
        L.sfb_mlr_sf_csr.argtypes = [vp, vp, i64, i64, ctypes.POINTER(sfb_csr), vp, vp]
        L.sfb_mlr_sf_csr.restype = ctypes.c_int
        L.sfb_set_csr_route.argtypes = [vp, ctypes.c_int]
        L.sfb_set_csr_route.restype = ctypes.c_int
        L.sfb_apply_csr_workspace_bytes.argtypes = [i64, i64, i64, i32]
        L.sfb_apply_csr_workspace_bytes.restype = i64
        L.sfb_apply_csr.argtypes = [vp, vp, i64, i64, vp, ctypes.POINTER(sfb_csr), vp, ctypes.c_float]
        L.sfb_apply_csr.restype = ctypes.c_int
        L.sfb_sdca_workspace_bytes.argtypes = [i64, i64, i64]
        L.sfb_sdca_workspace_bytes.restype = i64
        L.sfb_sdca_mlr_sf.argtypes = [vp, vp, i64, i64, vp, i64, vp, ctypes.c_float, i64, ctypes.c_float, vp]
        L.sfb_sdca_mlr_sf.restype = ctypes.c_int
        L.sfb_dual_to_primal_l2.argtypes = [vp, vp, vp, i64, i64, ctypes.c_float]
        L.sfb_dual_to_primal_l2.restype = ctypes.c_int
        pa, pr, pt = ctypes.POINTER(sfb_adapters), ctypes.POINTER(sfb_requests), ctypes.POINTER(sfb_tensor)
        for name in ("sfb_adapter_forward_workspace_bytes", "sfb_adapter_backward_workspace_bytes"):
            getattr(L, name).argtypes = [i64, i64, i64, pa]
            getattr(L, name).restype = i64
        L.sfb_adapter_forward.argtypes = [vp, vp, i32, i64, i64, vp, i64, pa, pr, vp, vp]
        L.sfb_adapter_forward.restype = ctypes.c_int
        L.sfb_adapter_backward.argtypes = [vp, vp, i32, i64, i64, vp, vp, i64, pa, pr, vp, vp, vp, vp]
        L.sfb_adapter_backward.restype = ctypes.c_int
        L.sfb_grad_norm_workspace_bytes.argtypes = [pt, i64]
        L.sfb_grad_norm_workspace_bytes.restype = i64
        L.sfb_tensor_table_bytes.argtypes = [i64]
        L.sfb_tensor_table_bytes.restype = i64
        L.sfb_tensor_table_fill.argtypes = [pt, i64, vp]
        L.sfb_tensor_table_fill.restype = ctypes.c_int
        L.sfb_grad_norm.argtypes = [vp, pt, i64, vp, vp]
        L.sfb_grad_norm.restype = ctypes.c_int
        L.sfb_clip_grads.argtypes = [vp, pt, i64, vp, ctypes.c_float, vp]
        L.sfb_clip_grads.restype = ctypes.c_int
        L.sfb_capturing.argtypes = [vp]
        L.sfb_capturing.restype = ctypes.c_int
        L.sfb_prox_rows.argtypes = [vp, vp, i64, i64, i32]
        L.sfb_prox_rows.restype = ctypes.c_int
        L.sfb_strerror.argtypes = [ctypes.c_int]
        L.sfb_strerror.restype = ctypes.c_char_p
        L.sfb_last_hip_error.argtypes = [vp]
        L.sfb_last_hip_error.restype = ctypes.c_int
        L.sfb_version.argtypes = []
        L.sfb_version.restype = ctypes.c_char_p
        L.sfb_profile_enable.argtypes = [vp, ctypes.c_int]
        L.sfb_profile_enable.restype = ctypes.c_int
        L.sfb_profile_collect.argtypes = [vp, ctypes.POINTER(sfb_kernel_time), ctypes.c_int,
                                          ctypes.POINTER(ctypes.c_int)]
        L.sfb_profile_collect.restype = ctypes.c_int
        L.sfb_set_wait_limit.argtypes = [vp, ctypes.c_int]
        L.sfb_set_wait_limit.restype = ctypes.c_int
        L.sfb_wait_fallbacks.argtypes = [vp, ctypes.POINTER(i64)]
        L.sfb_wait_fallbacks.restype = ctypes.c_int
        L.sfb_ssp_create.argtypes = [ctypes.POINTER(vp), i32, i32]
        L.sfb_ssp_create.restype = ctypes.c_int
        L.sfb_ssp_destroy.argtypes = [vp]
        L.sfb_ssp_destroy.restype = ctypes.c_int
        L.sfb_ssp_can_compute.argtypes = [vp, i32]
        L.sfb_ssp_can_compute.restype = ctypes.c_int
        L.sfb_ssp_computed.argtypes = [vp, i32]
        L.sfb_ssp_computed.restype = i64
        L.sfb_ssp_delivered.argtypes = [vp, i32, i32]
        L.sfb_ssp_delivered.restype = i64
        L.sfb_ssp_pop_apply.argtypes = [vp, i32, ctypes.POINTER(i32), ctypes.POINTER(i64)]
        L.sfb_ssp_pop_apply.restype = ctypes.c_int
        L.sfb_ssp_clock.argtypes = [vp, i32]
        L.sfb_ssp_clock.restype = i64
        L.sfb_ssp_tau.argtypes = [vp, i32, i32]
        L.sfb_ssp_tau.restype = i64
        L.sfb_ssp_arrived.argtypes = [vp, i32, i32]
        L.sfb_ssp_arrived.restype = i64
        L.sfb_ssp_max_staleness_seen.argtypes = [vp]
        L.sfb_ssp_max_staleness_seen.restype = i64
        _lib = L
    return _lib


def strerror(code: int) -> str:
    return lib().sfb_strerror(int(code)).decode()


def version() -> str:
    return lib().sfb_version().decode()


_DTYPE_CODES = {torch.float32: SFB_F32, torch.bfloat16: SFB_BF16}


def _dtype_code(t: torch.Tensor) -> int:
    code = _DTYPE_CODES.get(t.dtype)
    if code is None:
        raise TypeError("unsupported dtype %s" % t.dtype)
    return code


def _ptr(t, name, dtype=None, shape=None):
    # a plain tensor that passes every check below: nothing converted, one comparison each (a small step is bound by these)
    if (type(t) is torch.Tensor and t.is_cuda and t.is_contiguous() and (dtype is None or t.dtype is dtype)
            and (shape is None or t.shape == shape)):
        return t.data_ptr()
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("%s must be a device tensor" % name)
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous (dense row-major)" % name)
    if dtype is not None and t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError("%s must have shape %r, got %r" % (name, tuple(shape), tuple(t.shape)))
    return t.data_ptr()


class TensorList:
    """A list of tensors for sfb_grad_norm and sfb_clip_grads, made once (not while a graph is captured) and used for as long as
    the tensors keep their memory: `src` the gradients (fp32 or bf16, contiguous, any sizes), `dst` where the clipped ones go (None: in place)."""

    def __init__(self, src, dst=None):
        src = list(src)
        dst = src if dst is None else list(dst)
        if len(dst) != len(src):
            raise ValueError("src and dst must have the same number of tensors")
        self.tensors = (src, dst)        # (kept alive with the list)
        self.device = None
        self.items = (sfb_tensor * max(1, len(src)))()
        self.count = len(src)
        for k, (s, d) in enumerate(zip(src, dst)):
            item = self.items[k]
            item.src, item.n, item.dtype = _ptr(s, "src[%d]" % k), s.numel(), _dtype_code(s)
            item.dst = item.src if d is s else _ptr(d, "dst[%d]" % k, dtype=s.dtype, shape=tuple(s.shape))
            for t in (s, d):
                if self.device is None:
                    self.device = t.device
                elif t.device != self.device:
                    raise ValueError("the tensors of a list must be on one device")
        need = lib().sfb_grad_norm_workspace_bytes(self.items, self.count)
        if need < 0:
            raise SfbError(int(need), "sfb_grad_norm_workspace_bytes")
        self.workspace_bytes = int(need)
        self.disjoint = None             # whether they can be clipped (found by the first call that does)
        self.table, self.table_ptr = None, None
        if self.count > 160:             # more than a launch takes as its arguments: described in device memory
            host = torch.zeros(int(lib().sfb_tensor_table_bytes(self.count)), dtype=torch.uint8)
            rc = lib().sfb_tensor_table_fill(self.items, self.count, host.data_ptr())
            if rc != SFB_OK:
                raise SfbError(rc, "sfb_tensor_table_fill")
            self.table = host.to(self.device)        # (waits for the copy: any stream may use it)
            self.table_ptr = self.table.data_ptr()

    def can_clip(self):
        """Whether no tensor that clipping writes overlaps another one of the list."""
        if self.disjoint is None:
            size = {SFB_F32: 4, SFB_BF16: 2}
            spans = []
            for k in range(self.count):
                item = self.items[k]
                if item.n:
                    bytes_ = item.n * size[item.dtype]
                    spans.append((item.dst, item.dst + bytes_, True))
                    if item.src != item.dst:
                        spans.append((item.src, item.src + bytes_, False))
            spans.sort()
            end = end_written = 0
            self.disjoint = True
            for first, last, written in spans:
                if first < (end if written else end_written):
                    self.disjoint = False
                    break
                end = max(end, last)
                if written:
                    end_written = max(end_written, last)
        return self.disjoint


class Context:
    """One sfb_ctx bound to a device and a stream; owns a torch workspace tensor.  Graphs that captured its calls work in memory
    that it holds: keep it for as long as they are replayed, and let no two of them, nor one and a call, run at the same time."""

    def __init__(self, device=0, stream=None):
        self._h = ctypes.c_void_p()
        self.device = torch.device("cuda", device if isinstance(device, int) else torch.device(device).index or 0)
        if stream is None:
            stream = torch.cuda.current_stream(self.device)
        self.stream = stream
        rc = lib().sfb_create(ctypes.byref(self._h), self.device.index, ctypes.c_void_p(stream.cuda_stream))
        if rc != SFB_OK:
            raise SfbError(rc, "sfb_create")
        self._ws = None
        self._captured, self._retired = False, []      # whether a graph works in _ws; memory from before it that graphs work in
        self._tables = {}                              # and tables of lists that they read (by their ids)
        self._index, self._raw = self.device.index, stream.cuda_stream
        self._one_device = torch.cuda.device_count() == 1
        self._ad, self._rq, self._needs = sfb_adapters(), sfb_requests(), {}
        self._graphs = False                           # whether any call has been captured
        self._shadow = None                            # (W tensor, buffer tensor) of an attached matrix

    # -- the buffer of an attached matrix, on the context's stream -----------------
    def _attached_buffer(self, need):
        if self._shadow is not None and self._shadow[1].numel() >= need:
            return self._shadow[1]
        with torch.cuda.stream(self.stream):
            return torch.empty(need, dtype=torch.uint8, device=self.device)

    def _attached(self, W, buf):
        """A buffer that another one takes the place of stays as long as a captured graph may write to it."""
        self._graphs = self._graphs or self._capturing()
        if self._shadow is not None and self._shadow[1] is not buf and self._graphs:
            self._retired.append(self._shadow[1])
        self._shadow = None if W is None else (W, buf)          # (W tensor, buffer tensor)

    # -- bf16 working copy of W ----------------------------------------------
    def sfb_shadow_attach(self, W):
        """Allocates (once) and fills the bf16 working copy of W; call again to refresh it."""
        J, D = W.shape
        need = lib().sfb_shadow_bytes(J, D)
        if need < 0:
            raise SfbError(int(need), "sfb_shadow_bytes")
        buf = self._attached_buffer(need)
        self._check(lib().sfb_shadow_attach(self._h, _ptr(W, "W", dtype=torch.float32), J, D, buf.data_ptr(),
                                            buf.numel()), "sfb_shadow_attach")
        self._attached(W, buf)

    def sfb_shadow_detach(self):
        self._check(lib().sfb_shadow_detach(self._h), "sfb_shadow_detach")
        self._attached(None, None)

    # -- W kept as two 16-bit planes --------------------------------------------
    def sfb_split_attach(self, W):
        """Allocates (once) the two planes and converts W into them; from then on W's fp32 array is stale
        until sfb_split_export.  Call again to re-convert after changing W yourself."""
        J, D = W.shape
        need = lib().sfb_split_bytes(J, D)
        if need < 0:
            raise SfbError(int(need), "sfb_split_bytes")
        buf = self._attached_buffer(need)
        self._check(lib().sfb_split_attach(self._h, _ptr(W, "W", dtype=torch.float32), J, D, buf.data_ptr(),
                                           buf.numel()), "sfb_split_attach")
        self._attached(W, buf)

    def sfb_split_export(self, W):
        """Enqueues the write-back of the current parameters into W's fp32 array."""
        self._graphs = self._graphs or self._capturing()
        self._check(lib().sfb_split_export(self._h, _ptr(W, "W", dtype=torch.float32)), "sfb_split_export")

    def sfb_split_detach(self):
        self._check(lib().sfb_split_detach(self._h), "sfb_split_detach")
        self._attached(None, None)

    def close(self):
        if self._h:
            lib().sfb_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc, what):
        if rc != SFB_OK:
            raise SfbError(rc, what, lib().sfb_last_hip_error(self._h))

    # -- the bounded wait of the softmax of long rows ----------------------------
    def sfb_set_wait_limit(self, polls: int = -1):
        self._check(lib().sfb_set_wait_limit(self._h, int(polls)), "sfb_set_wait_limit")

    def sfb_wait_fallbacks(self) -> int:
        """Partner pairs workgroups computed themselves so far on this device (waits for the stream)."""
        n = ctypes.c_int64(0)
        self._check(lib().sfb_wait_fallbacks(self._h, ctypes.byref(n)), "sfb_wait_fallbacks")
        return int(n.value)

    # -- per-kernel timing ---------------------------------------------------
    def sfb_profile_enable(self, on=True):
        self._check(lib().sfb_profile_enable(self._h, 1 if on else 0), "sfb_profile_enable")

    def sfb_profile_collect(self):
        """Synchronises the stream; returns {kernel group: (launches, total_ms)} since the last collect."""
        buf = (sfb_kernel_time * 32)()
        n = ctypes.c_int(0)
        self._check(lib().sfb_profile_collect(self._h, buf, 32, ctypes.byref(n)), "sfb_profile_collect")
        return {buf[i].name.decode(): (int(buf[i].launches), float(buf[i].total_ms)) for i in range(n.value)}

    # -- workspace ---------------------------------------------------------
    def sfb_workspace_bytes(self, model, J, D, batch: sfb_batch) -> int:
        n = lib().sfb_workspace_bytes(model, J, D, ctypes.byref(batch))
        if n < 0:
            raise SfbError(int(n), "sfb_workspace_bytes")
        return int(n)

    def sfb_set_workspace(self, tensor):
        """Use `tensor` (uint8, device) as scratch; None clears it."""
        if tensor is None:
            self._check(lib().sfb_set_workspace(self._h, None, 0), "sfb_set_workspace")
        else:
            self._check(lib().sfb_set_workspace(self._h, tensor.data_ptr(), tensor.numel() * tensor.element_size()),
                        "sfb_set_workspace")
        old, self._ws = self._ws, tensor
        if old is not None and old is not tensor:
            if self._captured:
                self._retired.append(old)
                self._captured = False
            else:
                old.record_stream(self.stream)       # (it may belong to another one)

    def sfb_apply_workspace_bytes(self, J, D, N, sf_dtype) -> int:
        n = lib().sfb_apply_workspace_bytes(J, D, N, sf_dtype)
        if n < 0:
            raise SfbError(int(n), "sfb_apply_workspace_bytes")
        return int(n)

    def _capturing(self):
        """Whether the context's stream is being captured into a graph."""
        # (0.3 us of a small call's 7)
        if self._one_device and torch._C._cuda_getCurrentRawStream(self._index) == self._raw:
            return torch._C._cuda_isCurrentStreamCapturing()
        return lib().sfb_capturing(self._h) > 0

    def _grow_workspace(self, need):
        """Room for `need` bytes, allocated on the context's stream; every call that takes a workspace comes here.  What a captured
        graph works in stays allocated when the workspace is replaced: the graph replays on the old one."""
        if need > (0 if self._ws is None else self._ws.numel()):
            with torch.cuda.stream(self.stream):
                self.sfb_set_workspace(torch.empty(need, dtype=torch.uint8, device=self.device))
        if not self._captured and self._capturing():
            self._captured = self._graphs = True

    def _ensure_workspace(self, model, J, D, batch, W=None):
        need = self.sfb_workspace_bytes(model, J, D, batch)
        if (model == SFB_MLR and batch.in_dtype == SFB_BF16 and self._shadow is not None and W is not None
                and self._shadow[0].data_ptr() == W.data_ptr() and tuple(self._shadow[0].shape) == (J, D)):
            need -= lib().sfb_shadow_bytes(J, D)
        self._grow_workspace(need)

    # -- the calls of the path --------------------------------------------
    def sfb_compute_sf(self, model, W, X, Y=None, sim=None, U=None, V=None, n_active=None,
                       lam=0.1, ista_iters=20, power_iters=10, margin=1.0):
        """Enqueues the SF computation; U (and V) must be preallocated device tensors."""
        J, D = W.shape
        B = X.shape[0]
        b = sfb_batch()
        b.X = _ptr(X, "X", shape=(B, D))
        b.B = B
        b.in_dtype = _dtype_code(X)
        b.sf_dtype = _dtype_code(U)
        b.lambda_ = lam
        b.ista_iters = ista_iters
        b.power_iters = power_iters
        b.margin = margin
        if model == SFB_MLR:
            b.Y = _ptr(Y, "Y (labels)", dtype=torch.int32, shape=(B,))
        elif model == SFB_DML:
            b.Y = _ptr(Y, "Y", dtype=X.dtype, shape=(B, D))
            b.sim = _ptr(sim, "sim", dtype=torch.int8, shape=(B,))
        self._ensure_workspace(model, J, D, b, W)
        rc = lib().sfb_compute_sf(self._h, model, _ptr(W, "W", dtype=torch.float32), J, D, ctypes.byref(b),
                                  _ptr(U, "U", shape=(B, J)),
                                  _ptr(V, "V", shape=(B, D)) if V is not None else None,
                                  _ptr(n_active, "n_active", dtype=torch.int32) if n_active is not None else None)
        self._check(rc, "sfb_compute_sf")

    def sfb_apply(self, W, U, V, eta):
        """Enqueues W -= eta * U^T V (in place)."""
        J, D = W.shape
        N = U.shape[0]
        if U.dtype != V.dtype:
            raise TypeError("U and V must share a dtype")
        code = _dtype_code(U)
        self._grow_workspace(self.sfb_apply_workspace_bytes(J, D, N, code))
        rc = lib().sfb_apply(self._h, _ptr(W, "W", dtype=torch.float32), J, D, _ptr(U, "U", shape=(N, J)),
                             _ptr(V, "V", shape=(N, D)), N, code, float(eta))
        self._check(rc, "sfb_apply")

    def sfb_apply_static(self, W, U, V, eta):
        """sfb_apply on the library's static scratch: no workspace, nothing allocated (here or in the library)."""
        J, D = W.shape
        N = U.shape[0]
        if U.dtype != V.dtype:
            raise TypeError("U and V must share a dtype")
        self._graphs = self._graphs or self._capturing()
        rc = lib().sfb_apply_static(self._h, _ptr(W, "W", dtype=torch.float32), J, D, _ptr(U, "U", shape=(N, J)),
                                    _ptr(V, "V", shape=(N, D)), N, _dtype_code(U), float(eta))
        self._check(rc, "sfb_apply_static")

    def sfb_apply_signed(self, W, U, V, coef, eta):
        """Enqueues W -= eta * sum_i coef_i u_i v_i^T (in place); coef: fp32 device tensor [N]."""
        J, D = W.shape
        N = U.shape[0]
        if U.dtype != V.dtype:
            raise TypeError("U and V must share a dtype")
        need = lib().sfb_apply_signed_workspace_bytes(J, D, N, _dtype_code(U))
        if need < 0:
            raise SfbError(int(need), "sfb_apply_signed_workspace_bytes")
        self._grow_workspace(int(need))
        rc = lib().sfb_apply_signed(self._h, _ptr(W, "W", dtype=torch.float32), J, D, _ptr(U, "U", shape=(N, J)),
                                    _ptr(V, "V", shape=(N, D)), _ptr(coef, "coef", dtype=torch.float32, shape=(N,)),
                                    N, _dtype_code(U), float(eta))
        self._check(rc, "sfb_apply_signed")

    # -- CSR rows (samples / second factors) ----------------------------------
    @staticmethod
    def _csr(indptr, indices, values, cols):
        """sfb_csr over three device tensors: int64 [rows + 1], int32 [nnz], fp32 or bf16 [nnz]."""
        m = sfb_csr()
        rows = indptr.numel() - 1
        nnz = indices.numel()
        m.indptr = _ptr(indptr, "indptr", dtype=torch.int64)
        m.indices = _ptr(indices, "indices", dtype=torch.int32) if nnz else None
        m.values = _ptr(values, "values", shape=(nnz,)) if nnz else None
        m.rows, m.cols, m.nnz = rows, cols, nnz
        m.dtype = _dtype_code(values)
        return m

    def sfb_csr_check(self, indptr, indices, values, cols) -> int:
        """Number of format violations (waits for the stream)."""
        m = self._csr(indptr, indices, values, cols)
        self._grow_workspace(256)
        bad = ctypes.c_int64(0)
        self._check(lib().sfb_csr_check(self._h, ctypes.byref(m), ctypes.byref(bad)), "sfb_csr_check")
        return int(bad.value)

    def sfb_mlr_sf_csr(self, W, indptr, indices, values, y, U):
        """Enqueues U = softmax(W x_i) - onehot(y_i) for samples given as CSR rows."""
        J, D = W.shape
        m = self._csr(indptr, indices, values, D)
        B = m.rows
        need = lib().sfb_mlr_sf_csr_workspace_bytes(J, D, B, m.dtype)
        if need < 0:
            raise SfbError(int(need), "sfb_mlr_sf_csr_workspace_bytes")
        self._grow_workspace(int(need))
        if _dtype_code(U) != m.dtype:
            raise TypeError("U and the CSR values must share a dtype")
        rc = lib().sfb_mlr_sf_csr(self._h, _ptr(W, "W", dtype=torch.float32), J, D, ctypes.byref(m),
                                  _ptr(y, "y (labels)", dtype=torch.int32, shape=(B,)), _ptr(U, "U", shape=(B, J)))
        self._check(rc, "sfb_mlr_sf_csr")

    def sfb_set_csr_route(self, route: int = 0):
        """0: sfb_mlr_sf_csr picks its route per call; 1: dense product; 2: over the stored entries."""
        self._check(lib().sfb_set_csr_route(self._h, int(route)), "sfb_set_csr_route")

    def sfb_apply_csr(self, W, U, indptr, indices, values, eta, coef=None):
        """Enqueues W -= eta * sum_i coef_i u_i v_i^T with the v_i given as CSR rows (in place)."""
        J, D = W.shape
        m = self._csr(indptr, indices, values, D)
        N = m.rows
        if _dtype_code(U) != m.dtype:
            raise TypeError("U and the CSR values must share a dtype")
        need = lib().sfb_apply_csr_workspace_bytes(J, D, N, m.dtype)
        if need < 0:
            raise SfbError(int(need), "sfb_apply_csr_workspace_bytes")
        self._grow_workspace(int(need))
        rc = lib().sfb_apply_csr(self._h, _ptr(W, "W", dtype=torch.float32), J, D, _ptr(U, "U", shape=(N, J)),
                                 ctypes.byref(m),
                                 _ptr(coef, "coef", dtype=torch.float32, shape=(N,)) if coef is not None else None,
                                 float(eta))
        self._check(rc, "sfb_apply_csr")

    # -- SDCA on l2-regularised multiclass logistic regression ---------------
    def sfb_sdca_mlr_sf(self, W, X, P, lam, N, beta, dU):
        """Enqueues the dual coordinate steps of a mini-batch: dU = beta (p* - P), P += dU (in place)."""
        J, D = W.shape
        B = X.shape[0]
        need = lib().sfb_sdca_workspace_bytes(J, D, B)
        if need < 0:
            raise SfbError(int(need), "sfb_sdca_workspace_bytes")
        self._grow_workspace(int(need))
        rc = lib().sfb_sdca_mlr_sf(self._h, _ptr(W, "W", dtype=torch.float32), J, D,
                                   _ptr(X, "X", dtype=torch.float32, shape=(B, D)), B,
                                   _ptr(P, "P", dtype=torch.float32, shape=(B, J)), float(lam), int(N), float(beta),
                                   _ptr(dU, "dU", dtype=torch.float32, shape=(B, J)))
        self._check(rc, "sfb_sdca_mlr_sf")

    def sfb_dual_to_primal_l2(self, Z, W, lam):
        """Enqueues W = Z / lam."""
        J, D = W.shape
        rc = lib().sfb_dual_to_primal_l2(self._h, _ptr(Z, "Z", dtype=torch.float32, shape=(J, D)),
                                         _ptr(W, "W", dtype=torch.float32), J, D, float(lam))
        self._check(rc, "sfb_dual_to_primal_l2")

    # -- factor blocks beside a shared matrix -----------------------------------
    def _at(self, t, name, dtype, shape):
        """_ptr of a tensor that has to be on the context's device."""
        if (type(t) is torch.Tensor and t.is_cuda and t.get_device() == self._index and t.is_contiguous() and t.dtype is dtype
                and t.shape == shape):
            return t.data_ptr()
        p = _ptr(t, name, dtype=dtype, shape=shape)
        if p is None:
            raise TypeError("%s is missing" % name)
        if t.get_device() != self._index:
            raise ValueError("%s must be on %s, got %s" % (name, self.device, t.device))
        return p

    def _adapter_workspace(self, query, J, D, T, ad):
        key = (query, J, D, T, ad.count, ad.rank, ad.dtype)
        need = self._needs.get(key)
        if need is None:
            need = int(getattr(lib(), query)(J, D, T, ctypes.byref(ad)))
            if need < 0:
                raise SfbError(need, query)
            if len(self._needs) > 1000:
                self._needs.clear()
            self._needs[key] = need
        self._grow_workspace(need)

    def _adapters(self, W, X, start, adapter, U, V, ranks, scale):
        J, D = W.shape
        T = X.shape[0]
        if U.dim() != 3 or X.dim() != 2:
            raise ValueError("U and V must be [count][rank][...], X [T][D]")
        n, R, _ = U.shape
        dtype, ad, rq, at = X.dtype, self._ad, self._rq, self._at
        ad.count, ad.rank, ad.dtype = n, R, _dtype_code(X)
        ad.U = at(U, "U", dtype, (n, R, J))
        ad.V = at(V, "V", dtype, (n, R, D))
        ad.ranks = None if ranks is None else at(ranks, "ranks", torch.int32, (n,))
        ad.scale = None if scale is None else at(scale, "scale", torch.float32, (n,))
        S = adapter.numel()
        rq.start = at(start, "start", torch.int64, (S + 1,))
        rq.adapter = at(adapter, "adapter", torch.int32, (S,))
        rq.count = S
        return J, D, T, n, R, dtype, ad, rq, at(W, "W", W.dtype, (J, D)), at(X, "X", dtype, (T, D))

    def sfb_adapter_forward(self, W, X, start, adapter, U, V, Y, ranks=None, scale=None, H=None):
        """Enqueues Y = X W^T + H U_a (H = scale_a X V_a^T, written too where a tensor for it is given): rows
        start[q] .. start[q + 1] - 1 of X [T][D] with the factor block a = adapter[q] of U [n][R][J], V [n][R][D] (outside
        [0, n): none).  start int64 [S + 1] and adapter int32 [S] on the device; rows of no request stay as they are."""
        J, D, T, n, R, dtype, ad, rq, Wp, Xp = self._adapters(W, X, start, adapter, U, V, ranks, scale)
        self._adapter_workspace("sfb_adapter_forward_workspace_bytes", J, D, T, ad)
        Yp = self._at(Y, "Y", dtype, (T, J))
        if Yp == Xp and T:
            raise ValueError("Y must not be X: the call reads X while it writes")
        rc = lib().sfb_adapter_forward(self._h, Wp, _dtype_code(W), J, D, Xp, T, ad, rq, Yp,
                                       None if H is None else self._at(H, "H", torch.float32, (T, R)))
        self._check(rc, "sfb_adapter_forward")

    def sfb_adapter_backward(self, W, X, dY, start, adapter, U, V, dX=None, dU=None, dV=None, ranks=None, scale=None, H=None):
        """Enqueues the gradients of the forward call at dY [T][J]: dX of X's dtype, dU [n][R][J] and dV [n][R][D] fp32
        (None: not wanted).  H: what the forward call wrote, or None."""
        J, D, T, n, R, dtype, ad, rq, Wp, Xp = self._adapters(W, X, start, adapter, U, V, ranks, scale)
        self._adapter_workspace("sfb_adapter_backward_workspace_bytes", J, D, T, ad)
        at, f32 = self._at, torch.float32
        dYp, dXp = at(dY, "dY", dtype, (T, J)), None if dX is None else at(dX, "dX", dtype, (T, D))
        if T and (dXp == dYp or dXp == Xp):
            raise ValueError("dX must be neither dY nor X: the call reads them while it writes")
        rc = lib().sfb_adapter_backward(self._h, Wp, _dtype_code(W), J, D, Xp, dYp, T, ad, rq,
                                        None if H is None else at(H, "H", f32, (T, R)),
                                        dXp,
                                        None if dU is None else at(dU, "dU", f32, (n, R, J)),
                                        None if dV is None else at(dV, "dV", f32, (n, R, D)))
        self._check(rc, "sfb_adapter_backward")

    # -- norm and clipping of gradients ------------------------------------------
    def _list(self, tensors, norm):
        if tensors.device is not None and tensors.device != self.device:
            raise ValueError("the tensors must be on %s, got %s" % (self.device, tensors.device))
        self._grow_workspace(tensors.workspace_bytes)
        if tensors.table is not None:
            # the list may be gone before the kernels are, and its table belongs to the stream that was current when it was made
            if self._capturing():
                self._tables[id(tensors.table)] = tensors.table          # (every replay reads it)
            else:
                tensors.table.record_stream(self.stream)
        return self._at(norm, "norm", torch.float32, (1,))

    def sfb_grad_norm(self, tensors: TensorList, norm):
        """Enqueues norm[0] = the global 2-norm of the list's tensors."""
        p = self._list(tensors, norm)
        self._check(lib().sfb_grad_norm(self._h, tensors.items, tensors.count, tensors.table_ptr, p), "sfb_grad_norm")

    def sfb_clip_grads(self, tensors: TensorList, max_norm, norm):
        """Enqueues norm[0] and dst = src * min(1, max_norm / norm) for every tensor of the list."""
        p = self._list(tensors, norm)
        if not tensors.can_clip():
            raise ValueError("tensors that are clipped must not overlap (one of them listed twice?)")
        self._check(lib().sfb_clip_grads(self._h, tensors.items, tensors.count, tensors.table_ptr, float(max_norm), p), "sfb_clip_grads")

    def sfb_prox_rows(self, W, mode=SFB_PROX_PROJECT):
        J, D = W.shape
        self._graphs = self._graphs or self._capturing()
        self._check(lib().sfb_prox_rows(self._h, _ptr(W, "W", dtype=torch.float32), J, D, mode), "sfb_prox_rows")


class SspClock:
    """One sfb_ssp object (include/sfb_ssp.h): counters of BSP / SSP / ASP application of SF sets."""

    def __init__(self, P: int, s: int):
        self._h = ctypes.c_void_p()
        rc = lib().sfb_ssp_create(ctypes.byref(self._h), int(P), int(s))
        if rc != SFB_OK:
            raise SfbError(rc, "sfb_ssp_create")

    def close(self):
        if self._h:
            lib().sfb_ssp_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _chk(self, v, what):
        if v < 0:
            raise SfbError(int(v), what)
        return int(v)

    def sfb_ssp_can_compute(self, p: int) -> bool:
        return bool(self._chk(lib().sfb_ssp_can_compute(self._h, int(p)), "sfb_ssp_can_compute"))

    def sfb_ssp_computed(self, p: int) -> int:
        return self._chk(lib().sfb_ssp_computed(self._h, int(p)), "sfb_ssp_computed")

    def sfb_ssp_delivered(self, p: int, q: int) -> int:
        return self._chk(lib().sfb_ssp_delivered(self._h, int(p), int(q)), "sfb_ssp_delivered")

    def sfb_ssp_pop_apply(self, p: int):
        """(q, t) of the next SF set worker p has to apply now, or None."""
        q, t = ctypes.c_int32(), ctypes.c_int64()
        rc = self._chk(lib().sfb_ssp_pop_apply(self._h, int(p), ctypes.byref(q), ctypes.byref(t)), "sfb_ssp_pop_apply")
        return (q.value, t.value) if rc else None

    def sfb_ssp_clock(self, p: int) -> int:
        return self._chk(lib().sfb_ssp_clock(self._h, int(p)), "sfb_ssp_clock")

    def sfb_ssp_tau(self, p: int, q: int) -> int:
        return self._chk(lib().sfb_ssp_tau(self._h, int(p), int(q)), "sfb_ssp_tau")

    def sfb_ssp_arrived(self, p: int, q: int) -> int:
        return self._chk(lib().sfb_ssp_arrived(self._h, int(p), int(q)), "sfb_ssp_arrived")

    def sfb_ssp_max_staleness_seen(self) -> int:
        return self._chk(lib().sfb_ssp_max_staleness_seen(self._h), "sfb_ssp_max_staleness_seen")
