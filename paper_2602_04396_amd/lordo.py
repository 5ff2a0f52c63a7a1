"""Thin ctypes binding of liblordo.so (see include/lordo.h for the contract of every call).

Only argument marshalling happens here: torch tensors supply device memory and the
current stream; every step of the path runs in the library's kernels.  There is no
fallback: if the library has not been built, importing `load()` raises.
"""
from __future__ import annotations

import ctypes as C
import os
import struct

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "lib", "liblordo.so")

OK, EINVAL, ENOMEM, EHIP, ESTATE, ENUMERIC = 0, -1, -2, -3, -4, -5
F32, BF16, Q8, I32, I64 = 0, 1, 2, 3, 4
STATE_Q, STATE_U, STATE_V, STATE_ANCHOR, STATE_MOM, STATE_GLOW, STATE_NUPD, STATE_ERR, STATE_UPLINK, STATE_RITZ = range(10)

EXPORTS = [
    "lordo_workspace_bytes", "lordo_init", "lordo_local_step", "lordo_refresh_subspace",
    "lordo_export_pseudograd", "lordo_outer_step", "lordo_get_state", "lordo_set_state",
    "lordo_get_step", "lordo_set_step", "lordo_poll_status", "lordo_strerror", "lordo_destroy",
    "lordo_profile_enable", "lordo_profile_read", "lordo_get_mssv", "lordo_refresh_subspace_local",
    "lordo_export_uplink", "lordo_outer_step_lowrank", "lordo_init_projection", "lordo_sync_payload",
    "lordo_get_stable_rank", "lordo_spectral_gap", "lordo_init_static",
    "lordo_adamw_workspace_bytes", "lordo_adamw_init", "lordo_adamw_step", "lordo_adamw_sync_payload",
    "lordo_adamw_export_moments", "lordo_adamw_import_moments", "lordo_adamw_get_step", "lordo_adamw_set_step",
    "lordo_adamw_steps_taken", "lordo_adamw_poll_status", "lordo_adamw_destroy", "lordo_grad_norm",
    "lordo_embed_lookup", "lordo_embed_workspace_bytes", "lordo_embed_gradient", "lordo_embed_gradient_rows",
]
STATIC_WORKSPACE_BYTES = 64 << 20
NORM_WORKSPACE_BYTES = 8192
MAX_TOKENS, MAX_VOCAB = 1 << 25, 1 << 22
K_DOWN, K_ADAM, K_UP, K_OUTER, K_EXPORT, K_REFRESH = range(6)


class Shape(C.Structure):
    _fields_ = [("rows", C.c_int64), ("cols", C.c_int64), ("rank", C.c_int32), ("side", C.c_int32)]


class HParams(C.Structure):
    _fields_ = [
        ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double),
        ("bias_correction", C.c_int32), ("qhm_mode", C.c_int32),
        ("omega", C.c_double),
        ("error_feedback", C.c_int32), ("outer_nesterov", C.c_int32),
        ("outer_lr", C.c_double), ("outer_momentum", C.c_double),
        ("power_iters", C.c_int32), ("orth_passes", C.c_int32),
        ("grad_dtype", C.c_int32), ("uplink_buffer", C.c_int32),
        ("rayleigh_ritz", C.c_int32), ("param_dtype", C.c_int32),
        ("err_dtype", C.c_int32), ("reserved", C.c_int32),
        ("seed", C.c_uint64),
    ]


def hparams(beta1=0.9, beta2=0.999, eps=1e-8, bias_correction=True, outer_lr=1.0, outer_momentum=0.0,
            outer_nesterov=False, power_iters=2, orth_passes=2, grad_dtype=BF16, qhm_mode=0, omega=1.0,
            error_feedback=False, uplink_buffer=False, rayleigh_ritz=False, seed=0, param_dtype=F32, err_dtype=F32) -> HParams:
    return HParams(beta1, beta2, eps, int(bias_correction), qhm_mode, omega, int(error_feedback),
                   int(outer_nesterov), outer_lr, outer_momentum, power_iters, orth_passes, grad_dtype, int(uplink_buffer),
                   int(rayleigh_ritz), int(param_dtype), int(err_dtype), 0, int(seed))


class Tensor(C.Structure):
    _fields_ = [("rows", C.c_int64), ("cols", C.c_int64), ("decay", C.c_int32), ("reserved", C.c_int32)]


class Grad(C.Structure):
    _fields_ = [("data", C.c_void_p), ("index", C.c_void_p), ("rows", C.c_int64), ("cols", C.c_int64), ("slots", C.c_int64),
                ("dtype", C.c_int32), ("reserved", C.c_int32)]


class AdamWHParams(C.Structure):
    _fields_ = [("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double), ("weight_decay", C.c_double),
                ("bias_correction", C.c_int32), ("param_dtype", C.c_int32), ("state_dtype", C.c_int32), ("reserved", C.c_int32)]


def adamw_hparams(beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, bias_correction=True, param_dtype=F32, state_dtype=F32) -> AdamWHParams:
    return AdamWHParams(beta1, beta2, eps, weight_decay, int(bias_correction), int(param_dtype), int(state_dtype), 0)


class LordoError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"lordo error {code}: {msg}")
        self.code = code


_lib = None


def load() -> C.CDLL:
    """Load the built library; raise if it is missing (no CPU or eager fallback exists)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} not built: run `python -m paper_2602_04396_amd.build`")
    lib = C.CDLL(LIB_PATH)
    vp, vpp = C.c_void_p, C.POINTER(C.c_void_p)
    lib.lordo_workspace_bytes.argtypes = [C.POINTER(Shape), C.c_int32, C.POINTER(HParams), C.POINTER(C.c_size_t)]
    lib.lordo_init.argtypes = [C.POINTER(vp), C.POINTER(Shape), C.c_int32, C.POINTER(HParams), vp, C.c_size_t, vpp, vp]
    lib.lordo_init_static.argtypes = [C.POINTER(vp), C.POINTER(Shape), C.c_int32, C.POINTER(HParams), vpp, vp]
    lib.lordo_local_step.argtypes = [vp, vpp, vpp, C.c_double, C.c_double, vp]
    lib.lordo_refresh_subspace.argtypes = [vp, vpp, C.c_int32, vpp, vp]
    lib.lordo_refresh_subspace_local.argtypes = [vp, vpp, C.c_double, vpp, vp]
    lib.lordo_export_pseudograd.argtypes = [vp, vpp, vpp, vp]
    lib.lordo_outer_step.argtypes = [vp, vpp, vpp, vp]
    lib.lordo_init_projection.argtypes = [vp, vpp, vp]
    lib.lordo_export_uplink.argtypes = [vp, vpp, vp]
    lib.lordo_outer_step_lowrank.argtypes = [vp, vpp, vpp, vp]
    lib.lordo_sync_payload.argtypes = [vp, vpp, C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)]
    lib.lordo_get_state.argtypes = [vp, C.c_int32, C.c_int32, vp, vp]
    lib.lordo_set_state.argtypes = [vp, C.c_int32, C.c_int32, vp, vp]
    lib.lordo_get_mssv.argtypes = [vp, vp, vp]
    lib.lordo_get_stable_rank.argtypes = [vp, vp, vp]
    lib.lordo_spectral_gap.argtypes = [vp, vpp, C.c_int32, vpp, vp, vp]
    lib.lordo_get_step.argtypes = [vp, C.POINTER(C.c_int64)]
    lib.lordo_set_step.argtypes = [vp, C.c_int64]
    lib.lordo_poll_status.argtypes = [vp, vp]
    lib.lordo_profile_enable.argtypes = [vp, C.c_int32]
    lib.lordo_profile_read.argtypes = [vp, C.c_int32, C.POINTER(C.c_double), C.POINTER(C.c_int64), vp]
    lib.lordo_strerror.argtypes = [C.c_int]
    lib.lordo_strerror.restype = C.c_char_p
    lib.lordo_destroy.argtypes = [vp]
    lib.lordo_destroy.restype = None
    lib.lordo_adamw_workspace_bytes.argtypes = [C.POINTER(Tensor), C.c_int32, C.POINTER(AdamWHParams), C.POINTER(C.c_size_t)]
    lib.lordo_adamw_init.argtypes = [C.POINTER(vp), C.POINTER(Tensor), C.c_int32, C.POINTER(AdamWHParams), vp, C.c_size_t, vp]
    lib.lordo_adamw_step.argtypes = [vp, vpp, C.POINTER(Grad), C.c_double, C.c_double, vp, vp]
    lib.lordo_adamw_sync_payload.argtypes = [vp, vpp, C.POINTER(C.c_size_t)]
    lib.lordo_adamw_export_moments.argtypes = [vp, vp, vp]
    lib.lordo_adamw_import_moments.argtypes = [vp, vp, vp]
    lib.lordo_adamw_get_step.argtypes = [vp, C.POINTER(C.c_int64)]
    lib.lordo_adamw_set_step.argtypes = [vp, C.c_int64]
    lib.lordo_adamw_steps_taken.argtypes = [vp, C.POINTER(C.c_int64), vp]
    lib.lordo_adamw_poll_status.argtypes = [vp, vp]
    lib.lordo_adamw_destroy.argtypes = [vp]
    lib.lordo_adamw_destroy.restype = None
    lib.lordo_grad_norm.argtypes = [C.POINTER(Grad), C.c_int32, C.c_double, vp, vp, C.c_size_t, vp]
    i32, i64, f64, size = C.c_int32, C.c_int64, C.c_double, C.c_size_t
    lib.lordo_embed_lookup.argtypes = [vp, i32, i64, i64, vp, i32, i64, f64, vp, i32, vp]
    lib.lordo_embed_workspace_bytes.argtypes = [i64, i64, i64, C.POINTER(C.c_size_t)]
    lib.lordo_embed_gradient.argtypes = [vp, i32, i64, vp, i32, i64, i64, f64, i64, i32, vp, i32, vp, size, vp]
    lib.lordo_embed_gradient_rows.argtypes = [vp, i32, i64, vp, i32, i64, i64, f64, i64, vp, i32, vp, vp, size, vp]
    for name in EXPORTS:
        if name not in ("lordo_strerror", "lordo_destroy", "lordo_adamw_destroy"):
            getattr(lib, name).restype = C.c_int
    _lib = lib
    return lib


def _check(code):
    if code != OK:
        raise LordoError(code, load().lordo_strerror(code).decode())


class PtrList:
    """Pointer array of an already validated tensor list, reusable across calls (keeps the
    tensors alive).  Built by Lordo.ptrs() and AdamW.ptrs() (`made_for`: its shapes, type and
    device); lets a tight loop skip per-call validation."""

    def __init__(self, tensors, arr, made_for=None):
        self.tensors = tensors
        self.arr = arr
        self.made_for = made_for


def _ptr_array(tensors):
    if isinstance(tensors, PtrList):
        return tensors.arr
    arr = (C.c_void_p * len(tensors))()
    for i, t in enumerate(tensors):
        arr[i] = None if t is None else t.data_ptr()
    return arr


def _shape_array(shapes):
    arr = (Shape * len(shapes))()
    for i, sh in enumerate(shapes):      # (p, q, r) or (p, q, r, side); side 1 = projection on the right
        arr[i] = Shape(sh[0], sh[1], sh[2], sh[3] if len(sh) > 3 else 0)
    return arr


def workspace_bytes(shapes, hp: HParams) -> int:
    out = C.c_size_t(0)
    _check(load().lordo_workspace_bytes(_shape_array(shapes), len(shapes), C.byref(hp), C.byref(out)))
    return out.value


class Lordo:
    """One optimizer context over a list of (p, q, r) matrices.  `W` and every other
    argument is a list of torch CUDA tensors, contiguous, in the order of `shapes`."""

    def __init__(self, shapes, hp: HParams, W, torch, static_workspace=False):
        self.lib = load()
        self.torch = torch
        self.shapes = [tuple(s) for s in shapes]
        self.hp = hp
        self.n = len(shapes)
        self._check_tensors(W, torch.bfloat16 if hp.param_dtype == BF16 else torch.float32, "pq")
        self.device = W[0].device
        self.ctx = C.c_void_p()
        if static_workspace:         # lordo_init_static: the workspace is the library's own fixed array, nothing is allocated
            self.arena = None
            _check(self.lib.lordo_init_static(C.byref(self.ctx), _shape_array(self.shapes), self.n, C.byref(hp),
                                              _ptr_array(W), self._stream()))
            return
        nbytes = workspace_bytes(self.shapes, hp)
        self.arena = torch.empty(nbytes + 256, dtype=torch.uint8, device=W[0].device)
        base = self.arena.data_ptr()
        self.arena_ptr = (base + 255) // 256 * 256
        self.arena_bytes = nbytes
        _check(self.lib.lordo_init(C.byref(self.ctx), _shape_array(self.shapes), self.n, C.byref(hp),
                                   C.c_void_p(self.arena_ptr), nbytes, _ptr_array(W), self._stream()))

    # -- helpers ----------------------------------------------------------------------------
    def _stream(self):
        return C.c_void_p(self.torch.cuda.current_stream().cuda_stream)

    def ptrs(self, tensors, dtype=None, kind="pq") -> PtrList:
        """Validate a tensor list once and freeze its device pointers for repeated calls."""
        self._check_tensors(tensors, dtype or self.torch.float32, kind)
        return PtrList(list(tensors), _ptr_array(tensors))

    def _check_tensors(self, ts, dtype, kind, allow_none=False):
        if isinstance(ts, PtrList):
            if ts.made_for is not None or len(ts.tensors) != self.n:      # AdamW's, or another set's: the library reads n pointers
                raise ValueError("a list of tensors made for other shapes")
            return
        if len(ts) != self.n:
            raise ValueError("one tensor per matrix expected")
        for t, sh in zip(ts, self.shapes):
            if t is None and allow_none:
                continue
            p, q, r = sh[:3]
            # low-rank arrays of a right-projected matrix are those of the transposed problem
            tp, tq = (q, p) if len(sh) > 3 and sh[3] else (p, q)
            want = {"pq": (p, q), "qr": (tq, r), "rq": (r, tq), "pr": (tp, r)}[kind]
            if tuple(t.shape) != want or t.dtype != dtype or not t.is_contiguous() or not t.is_cuda:
                raise ValueError(f"expected contiguous CUDA {dtype} tensor of shape {want}, got {t.dtype} {tuple(t.shape)}")

    def _w_dtype(self):
        return self.torch.bfloat16 if self.hp.param_dtype == BF16 else self.torch.float32

    def _grad_dtype(self):
        return self.torch.bfloat16 if self.hp.grad_dtype == BF16 else self.torch.float32

    # -- the four calls -----------------------------------------------------------------------
    def local_step(self, W, G, lr, grad_scale=1.0):
        self._check_tensors(W, self._w_dtype(), "pq")
        self._check_tensors(G, self._grad_dtype(), "pq")
        _check(self.lib.lordo_local_step(self.ctx, _ptr_array(W), _ptr_array(G), float(lr), float(grad_scale), self._stream()))

    def init_projection(self, block=None):
        """Q_0 = orthonormal basis of the p x r blocks given (Alg. 1: random initial projection); None: blocks
        drawn by the library from hp.seed."""
        if block is None:
            _check(self.lib.lordo_init_projection(self.ctx, None, self._stream()))
            return
        self._check_tensors(block, self.torch.float32, "pr")
        _check(self.lib.lordo_init_projection(self.ctx, _ptr_array(block), self._stream()))

    def refresh_subspace(self, Src, Omega=None):
        """Src: one tensor per matrix (None entries leave that matrix out); Omega None: start blocks from hp.seed."""
        src_list = Src.tensors if isinstance(Src, PtrList) else Src
        live = [t for t in src_list if t is not None]
        if not live:
            return
        dt = live[0].dtype
        if dt not in (self.torch.bfloat16, self.torch.float32):
            raise ValueError("refresh source must be bf16 or fp32")
        self._check_tensors(Src, dt, "pq", allow_none=True)
        if Omega is not None:
            self._check_tensors(Omega, self.torch.float32, "qr", allow_none=True)
        code = BF16 if dt == self.torch.bfloat16 else F32
        _check(self.lib.lordo_refresh_subspace(self.ctx, _ptr_array(Src), code, None if Omega is None else _ptr_array(Omega),
                                               self._stream()))

    def spectral_gap(self, Src, Omega):
        """Per matrix: estimate of sigma_r - sigma_{r+1} of Src (the source of the last refresh; needs rayleigh_ritz)."""
        dt = (Src.tensors if isinstance(Src, PtrList) else Src)[0].dtype
        if dt not in (self.torch.bfloat16, self.torch.float32):
            raise ValueError("source must be bf16 or fp32")
        self._check_tensors(Src, dt, "pq")
        self._check_tensors(Omega, self.torch.float32, "qr")
        out = self.torch.empty(len(self.shapes), dtype=self.torch.float32, device=self.device)
        _check(self.lib.lordo_spectral_gap(self.ctx, _ptr_array(Src), BF16 if dt == self.torch.bfloat16 else F32,
                                           _ptr_array(Omega), C.c_void_p(out.data_ptr()), self._stream()))
        return out

    def refresh_subspace_local(self, G, Omega, grad_scale=1.0):
        """Alg. 2 refresh from grad_scale * G + E; the next call must be local_step with the same G."""
        self._check_tensors(G, self._grad_dtype(), "pq")
        if Omega is not None:
            self._check_tensors(Omega, self.torch.float32, "qr")
        _check(self.lib.lordo_refresh_subspace_local(self.ctx, _ptr_array(G), float(grad_scale),
                                                     None if Omega is None else _ptr_array(Omega), self._stream()))

    def export_pseudograd(self, W, out):
        self._check_tensors(W, self._w_dtype(), "pq")
        self._check_tensors(out, self.torch.float32, "pq")
        _check(self.lib.lordo_export_pseudograd(self.ctx, _ptr_array(W), _ptr_array(out), self._stream()))

    def outer_step(self, W, avg_delta=None):
        self._check_tensors(W, self._w_dtype(), "pq")
        if avg_delta is not None:
            self._check_tensors(avg_delta, self.torch.float32, "pq")
            _check(self.lib.lordo_outer_step(self.ctx, _ptr_array(W), _ptr_array(avg_delta), self._stream()))
        else:
            _check(self.lib.lordo_outer_step(self.ctx, _ptr_array(W), None, self._stream()))

    def export_uplink(self, out):
        """out_i <- the r x q up-link buffer of matrix i (App. A.5.1)."""
        self._check_tensors(out, self.torch.float32, "rq")
        _check(self.lib.lordo_export_uplink(self.ctx, _ptr_array(out), self._stream()))

    def outer_step_lowrank(self, W, avg_acc=None):
        """Outer step with Delta = Q avg_acc (avg_acc: mean of the workers' exported buffers; None: own buffer)."""
        self._check_tensors(W, self._w_dtype(), "pq")
        if avg_acc is not None:
            self._check_tensors(avg_acc, self.torch.float32, "rq")
            _check(self.lib.lordo_outer_step_lowrank(self.ctx, _ptr_array(W), _ptr_array(avg_acc), self._stream()))
        else:
            _check(self.lib.lordo_outer_step_lowrank(self.ctx, _ptr_array(W), None, self._stream()))

    def sync_payload(self):
        """(payload, moments_count): the contiguous fp32 region [u | v | A] of the workspace as a tensor view
        (Alg. 1 synchronisation; App. A.5.1) and the number of leading elements that are moments."""
        if self.arena is None:
            raise ValueError("the payload view needs a torch-owned arena (context created with static_workspace)")
        ptr, count, moments = C.c_void_p(), C.c_size_t(), C.c_size_t()
        _check(self.lib.lordo_sync_payload(self.ctx, C.byref(ptr), C.byref(count), C.byref(moments)))
        off = ptr.value - self.arena.data_ptr()
        assert 0 <= off and off + 4 * count.value <= self.arena.numel()
        return self.arena[off:off + 4 * count.value].view(self.torch.float32), moments.value

    # -- state ------------------------------------------------------------------------------------
    def _state_shape(self, mat, which):
        sh = self.shapes[mat]
        p, q, r = sh[:3]
        tp, tq = (q, p) if len(sh) > 3 and sh[3] else (p, q)
        return {STATE_Q: (tp, r), STATE_ANCHOR: (p, q), STATE_MOM: (p, q), STATE_ERR: (p, q), STATE_RITZ: (r,)}.get(which, (r, tq))

    def get_state(self, mat, which):
        out = self.torch.empty(self._state_shape(mat, which), dtype=self.torch.float32, device=self.device)
        _check(self.lib.lordo_get_state(self.ctx, mat, which, C.c_void_p(out.data_ptr()), self._stream()))
        return out

    def set_state(self, mat, which, src):
        want = self._state_shape(mat, which)
        if tuple(src.shape) != want or src.dtype != self.torch.float32 or not src.is_contiguous() or not src.is_cuda:
            raise ValueError(f"expected contiguous CUDA float32 tensor of shape {want}")
        _check(self.lib.lordo_set_state(self.ctx, mat, which, C.c_void_p(src.data_ptr()), self._stream()))

    def mssv(self):
        """Per matrix: mean squared singular value of Q_new^T Q_old of the last refresh (tensor of n floats)."""
        out = self.torch.empty(len(self.shapes), dtype=self.torch.float32, device=self.device)
        _check(self.lib.lordo_get_mssv(self.ctx, C.c_void_p(out.data_ptr()), self._stream()))
        return out

    def stable_rank(self):
        """Per matrix: ||Src||_F^2 / ||Src||_2^2 of the source of the last refresh (needs rayleigh_ritz)."""
        out = self.torch.empty(len(self.shapes), dtype=self.torch.float32, device=self.device)
        _check(self.lib.lordo_get_stable_rank(self.ctx, C.c_void_p(out.data_ptr()), self._stream()))
        return out

    @property
    def step(self):
        t = C.c_int64(0)
        _check(self.lib.lordo_get_step(self.ctx, C.byref(t)))
        return t.value

    @step.setter
    def step(self, t):
        _check(self.lib.lordo_set_step(self.ctx, int(t)))

    def poll_status(self):
        _check(self.lib.lordo_poll_status(self.ctx, self._stream()))

    def profile_enable(self, on=True):
        _check(self.lib.lordo_profile_enable(self.ctx, int(on)))

    def profile_read(self, kernel_class):
        """(total milliseconds, number of spans) of one kernel class since profiling was enabled."""
        ms, cnt = C.c_double(0), C.c_int64(0)
        _check(self.lib.lordo_profile_read(self.ctx, kernel_class, C.byref(ms), C.byref(cnt), self._stream()))
        return ms.value, cnt.value

    def close(self):
        if self.ctx:
            self.lib.lordo_destroy(self.ctx)
            self.ctx = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---- what a model has beside its projected matrices: AdamW, gradient norm, token embedding ------------------------------

_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def _same_device(torch, *tensors):
    """The current GPU, where all tensors have to be: the calls without a context enqueue there."""
    at = torch.cuda.current_device() if tensors[0].is_cuda else -1
    for t in tensors:
        if t.get_device() != at or at < 0:
            raise ValueError("expected CUDA tensors on the current device, got " + ", ".join(str(t.device) for t in tensors))
    return at


def _stream_of(torch, at=None):
    """Address of the current stream of GPU `at` (the current one).  torch's own look-up takes 0.1 us, the Stream object of its public call 2.6."""
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if raw is None:
        return torch.cuda.current_stream().cuda_stream
    return raw(torch.cuda.current_device() if at is None else at)


def _float_code(t, torch):
    dtype = t.dtype
    if dtype is torch.float32:
        return F32
    if dtype is torch.bfloat16:
        return BF16
    raise ValueError(f"expected a float32 or bfloat16 tensor, got {dtype}")


def _rows_cols(t):
    return (t.shape[0], t.shape[1]) if t.dim() == 2 else (1, t.numel())


class RowGrad:
    """Gradient of a (vocab, cols) tensor by rows, as embed_gradient_rows returns it: `rows` (slots, cols), `index` int32 (vocab + slots): the row of
    `rows` of each row of the tensor, or -1, and behind them the row of the tensor of each row of `rows`, or -1.  `rows` holds nothing where that is -1."""

    def __init__(self, rows, index, vocab):
        if rows.dim() != 2 or index.dim() != 1 or index.numel() != vocab + rows.shape[0] or index.dtype != _torch().int32:
            raise ValueError("expected rows (slots, cols) and an int32 index of vocab + slots")
        self.rows, self.index, self.vocab = rows, index, vocab

    @property
    def shape(self):
        return (self.vocab, self.rows.shape[1])


_float_codes = {}


class GradList:
    """A list of gradients (tensors of one or two dimensions, RowGrads) validated once, reusable across calls; keeps them alive."""

    def __init__(self, grads):
        codes = _float_codes
        if not codes:
            torch = _torch()
            codes.update({torch.float32: F32, torch.bfloat16: BF16})
        self.grads = grads = list(grads)
        if not grads:
            raise ValueError("no gradients")
        first = grads[0].rows if type(grads[0]) is RowGrad else grads[0]
        self.at, self.device = at, _ = first.get_device(), first.device
        fields = []
        for g in grads:
            index = slots = 0
            if type(g) is RowGrad:
                index, slots, vocab, same = g.index.data_ptr(), len(g.rows), g.vocab, g.index.get_device() == at and g.index.is_contiguous()
                g = g.rows
                rows, cols = vocab, g.shape[1]
            else:
                same = True
                shape = g.shape
                rows, cols = shape if len(shape) == 2 else (1, g.numel())
            code = codes.get(g.dtype)
            if code is None or not g.is_contiguous() or not same or g.get_device() != at or at < 0:
                raise ValueError(f"expected contiguous float32 or bfloat16 CUDA tensors on one device, got {g.dtype} on {g.device}")
            fields += (g.data_ptr(), index, rows, cols, slots, code, 0)
        self.arr = (Grad * len(grads)).from_buffer_copy(struct.pack("QQqqqii" * len(grads), *fields))

    def __len__(self):
        return len(self.grads)


def grad_list(grads) -> GradList:
    return grads if isinstance(grads, GradList) else GradList(grads)


def grad_norm(grads, max_norm=float("inf"), out=None):
    """Tensor of two floats on the device: the norm over all gradients, and min(1, max_norm / norm) (Alg. 1 clip; NaN if the norm is not finite).
    AdamW.local_step takes it as `clip`; Lordo.local_step takes its second value, read back, as grad_scale."""
    torch = _torch()
    if not isinstance(grads, GradList):
        grads = GradList(grads)
    gpu = torch.cuda.current_device()
    if grads.at != gpu:
        raise ValueError(f"tensors are on {grads.device}, which is not the current device")
    # the result and, from 256 bytes on, the workspace in one allocation
    room = torch.empty(64 + NORM_WORKSPACE_BYTES // 4, dtype=torch.float32, device=grads.device)
    at = room.data_ptr()
    if out is None:
        out = room[:2]
    elif out.dtype != torch.float32 or out.numel() != 2 or not out.is_contiguous() or out.device != grads.device:
        raise ValueError("expected a contiguous float32 tensor of two elements on the gradients' device")
    _check(load().lordo_grad_norm(grads.arr, len(grads.grads), max_norm, out.data_ptr(), at + 256, NORM_WORKSPACE_BYTES, _stream_of(torch, gpu)))
    return out


class AdamW:
    """AdamW over the tensors that are not projected.  `shapes`: (rows, cols) or (rows, cols, decay) of each, a vector as (1, cols); `W` is a list of
    torch CUDA tensors of those sizes, contiguous, of hp.param_dtype; gradients are tensors or RowGrads."""

    def __init__(self, shapes, hp: AdamWHParams, torch, device=None):
        self.lib, self.torch, self.hp = load(), torch, hp
        self.ctx = C.c_void_p()
        self.shapes = [tuple(sh) for sh in shapes]
        current = torch.device("cuda", torch.cuda.current_device())
        self.device = current if device is None else torch.device(device)
        if self.device == torch.device("cuda"):          # ("cuda" without a number: the current one)
            self.device = current
        self.made_for = (self.device, hp.param_dtype, tuple(sh[:2] for sh in self.shapes))
        self.at = self.device.index
        if self.device != current:
            raise ValueError(f"{self.device} is not the current device")
        arr = (Tensor * len(self.shapes))()
        for a, sh in zip(arr, self.shapes):
            a.rows, a.cols, a.decay = sh[0], sh[1], sh[2] if len(sh) > 2 else 1
        nbytes = C.c_size_t(0)
        _check(self.lib.lordo_adamw_workspace_bytes(arr, len(arr), C.byref(hp), C.byref(nbytes)))
        self.arena = torch.empty(nbytes.value + 256, dtype=torch.uint8, device=self.device)
        base = (self.arena.data_ptr() + 255) // 256 * 256
        _check(self.lib.lordo_adamw_init(C.byref(self.ctx), arr, len(arr), C.byref(hp), C.c_void_p(base), nbytes.value, self._stream()))

    def _stream(self):
        return _stream_of(self.torch)

    def ptrs(self, W) -> PtrList:
        """Validate the list of weights once and freeze its pointers for repeated calls."""
        if isinstance(W, PtrList):
            if W.made_for != self.made_for:
                raise ValueError("a list of weights made for other shapes")
            return W
        dtype = self.torch.bfloat16 if self.hp.param_dtype == BF16 else self.torch.float32
        if len(W) != len(self.shapes):
            raise ValueError("one tensor per shape expected")
        for t, sh in zip(W, self.shapes):
            if _rows_cols(t) != sh[:2] or t.dtype != dtype or not t.is_contiguous() or t.device != self.device:
                raise ValueError(f"expected a contiguous {dtype} tensor of shape {sh[:2]} on {self.device}, got {t.dtype} {tuple(t.shape)} on {t.device}")
        spans = sorted((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in W)
        if any(a[1] > b[0] for a, b in zip(spans, spans[1:])):
            raise ValueError("two of the weights overlap: a tensor is stepped once")
        return PtrList(list(W), _ptr_array(W), self.made_for)

    def local_step(self, W, G, lr, grad_scale=1.0, clip=None):
        """One step; the gradient is grad_scale * clip[1] * G (clip: what grad_norm returned, or None)."""
        if getattr(W, "made_for", None) is not self.made_for:
            W = self.ptrs(W)
        if not isinstance(G, GradList):
            G = GradList(G)
        if len(G.grads) != len(self.shapes) or G.at != self.at:
            raise ValueError(f"expected one gradient per shape on {self.device}")
        at = None
        if clip is not None:
            if clip.dtype is not self.torch.float32 or clip.numel() != 2 or not clip.is_contiguous() or clip.get_device() != self.at:
                raise ValueError("clip: expected the two floats of grad_norm")
            at = clip.data_ptr()
        _check(self.lib.lordo_adamw_step(self.ctx, W.arr, G.arr, lr, grad_scale, at, _stream_of(self.torch)))

    def _moments(self):
        ptr, count = C.c_void_p(), C.c_size_t()
        _check(self.lib.lordo_adamw_sync_payload(self.ctx, C.byref(ptr), C.byref(count)))
        return ptr.value, count.value

    def sync_payload(self):
        """The moments [u | v] in the arena as a (2, n) fp32 view (Alg. 1 synchronisation); tensor i starts at a multiple of 128 elements, in the order of
        the shapes.  Moments in 8 bits have none: export_moments, import_moments."""
        ptr, count = self._moments()
        if ptr is None:
            raise ValueError("moments in 8 bits have no fp32 array: use export_moments and import_moments")
        off = ptr - self.arena.data_ptr()
        return self.arena[off:off + 4 * count].view(self.torch.float32).view(2, -1)

    def _check_moments(self, t, count):
        if t.dtype != self.torch.float32 or t.numel() != count or not t.is_contiguous() or t.device != self.device:
            raise ValueError(f"expected a contiguous float32 tensor of {count} elements on {self.device}")

    def export_moments(self, out=None):
        count = self._moments()[1]
        if out is None:
            out = self.torch.empty((2, count // 2), dtype=self.torch.float32, device=self.device)
        self._check_moments(out, count)
        _check(self.lib.lordo_adamw_export_moments(self.ctx, C.c_void_p(out.data_ptr()), self._stream()))
        return out

    def import_moments(self, src):
        self._check_moments(src, self._moments()[1])
        _check(self.lib.lordo_adamw_import_moments(self.ctx, C.c_void_p(src.data_ptr()), self._stream()))

    @property
    def step(self):
        t = C.c_int64(0)
        _check(self.lib.lordo_adamw_get_step(self.ctx, C.byref(t)))
        return t.value

    @step.setter
    def step(self, t):
        _check(self.lib.lordo_adamw_set_step(self.ctx, int(t)))

    def steps_taken(self):
        """Steps that the device has counted, replays among them and steps left out not (`step` counts the calls): what to save beside the moments
        and to set `step` to when a run goes on from them.  Synchronises."""
        t = C.c_int64(0)
        _check(self.lib.lordo_adamw_steps_taken(self.ctx, C.byref(t), self._stream()))
        return t.value

    def poll_status(self):
        """Raises (ENUMERIC) if a step was left out since the last poll because the clip coefficient, or grad_scale times it, was not finite."""
        _check(self.lib.lordo_adamw_poll_status(self.ctx, self._stream()))

    def close(self):
        if self.ctx:
            self.lib.lordo_adamw_destroy(self.ctx)
            self.ctx = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _ids(ids, torch):
    """Address, type code and number of token ids."""
    dtype = ids.dtype
    if (dtype is not torch.int64 and dtype is not torch.int32) or not ids.is_contiguous():
        raise ValueError("expected contiguous int32 or int64 token ids")
    return ids.data_ptr(), I64 if dtype is torch.int64 else I32, ids.numel()


def embed_lookup(table, ids, scale=1.0, out=None, dtype=None):
    """out[...] = scale * table[ids[...]] as a tensor of ids.shape + (cols,), of `dtype` (the table's if None); zeros for ids outside [0, vocab).
    Autograd does not see it, also where the table requires a gradient: the output has none, its gradient goes to embed_gradient or embed_gradient_rows."""
    torch = _torch()
    if table.dim() != 2 or not table.is_contiguous():
        raise ValueError("expected a contiguous (vocab, cols) table")
    p, code, n = _ids(ids, torch)
    vocab, cols = table.shape
    if out is None:
        out = torch.empty((*ids.shape, cols), dtype=dtype or table.dtype, device=table.device)
    elif tuple(out.shape) != (*ids.shape, cols) or not out.is_contiguous() or (dtype is not None and out.dtype != dtype):
        raise ValueError(f"expected a contiguous output of shape {(*ids.shape, cols)}")
    at = _same_device(torch, table, ids, out)
    _check(load().lordo_embed_lookup(table.data_ptr(), _float_code(table, torch), vocab, cols, p, code, n, scale, out.data_ptr(),
                                     _float_code(out, torch), _stream_of(torch, at)))
    return out


def _workspace(ids, dy, vocab, torch):
    """Columns of dy, and bytes and tensor of the workspace of its gradient."""
    cols = dy.shape[-1]
    if dy.shape[:-1] != ids.shape or not dy.is_contiguous():
        raise ValueError(f"expected a contiguous gradient of shape {(*ids.shape, cols)}")
    size = C.c_size_t(0)
    _check(load().lordo_embed_workspace_bytes(ids.numel(), vocab, cols, C.byref(size)))
    return cols, size.value, torch.empty(size.value, dtype=torch.uint8, device=dy.device)


def embed_gradient(ids, dy, out, scale=1.0, pad_id=-1, accumulate=False):
    """Dense gradient of embed_lookup: out (vocab, cols) <- scale * sum of dy over the tokens of each row, added to out with accumulate."""
    torch = _torch()
    if out.dim() != 2 or not out.is_contiguous() or dy.shape[-1] != out.shape[1]:
        raise ValueError("expected a contiguous (vocab, cols) output")
    at = _same_device(torch, ids, dy, out)
    p, code, n = _ids(ids, torch)
    cols, size, ws = _workspace(ids, dy, out.shape[0], torch)
    _check(load().lordo_embed_gradient(p, code, n, dy.data_ptr(), _float_code(dy, torch), out.shape[0], cols, scale, pad_id, int(accumulate),
                                       out.data_ptr(), _float_code(out, torch), ws.data_ptr(), size, _stream_of(torch, at)))
    return out


def embed_gradient_rows(ids, dy, vocab, scale=1.0, pad_id=-1, dtype=None, out=None) -> RowGrad:
    """Gradient of embed_lookup by rows, for AdamW.local_step and grad_norm: one row per different token, of `dtype` (float32 if None).  `out`: an
    earlier result for as many tokens to write over, so that a GradList that holds it stays good."""
    torch = _torch()
    at = _same_device(torch, ids, dy)
    p, code, n = _ids(ids, torch)
    cols, size, ws = _workspace(ids, dy, vocab, torch)
    if out is None:
        rows = torch.empty((n, cols), dtype=dtype or torch.float32, device=dy.device)
        index = torch.empty(vocab + n, dtype=torch.int32, device=dy.device)
        out = RowGrad(rows, index, vocab)
    else:
        rows, index = out.rows, out.index
        if out.vocab != vocab or rows.shape != (n, cols) or (dtype is not None and rows.dtype != dtype) or not rows.is_contiguous() or not index.is_contiguous():
            raise ValueError(f"expected a RowGrad of {n} rows of {cols} for {vocab} ids")
        _same_device(torch, rows, index)
    _check(load().lordo_embed_gradient_rows(p, code, n, dy.data_ptr(), _float_code(dy, torch), vocab, cols, scale, pad_id, rows.data_ptr(),
                                            _float_code(rows, torch), index.data_ptr(), ws.data_ptr(), size, _stream_of(torch, at)))
    return out
