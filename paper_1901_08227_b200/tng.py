"""ctypes binding of libtng.so.  Names mirror ``include/tng.h``; the wrappers only
marshal arguments (tensor -> device pointer, current CUDA stream -> void*)."""
from __future__ import annotations

import ctypes as C
import functools
from pathlib import Path

import torch

_PKG = Path(__file__).resolve().parent
LIB_PATH = _PKG / "libtng.so"

CODEC_SIGN1, CODEC_TERN2, CODEC_QSGD4 = 1, 2, 4
NORM_NONE, NORM_DIFF, NORM_QUOT, NORM_COMB, NORM_MEAN = 0, 1, 2, 3, 4
SCALE_ABSMAX, SCALE_L2 = 0, 1
FUSE_AUTO, FUSE_LAST, FUSE_MEAN, FUSE_LSQ, FUSE_HINDSIGHT = 0, 1, 2, 3, 4
(OPT_BLOCK, OPT_QSGD_LEVELS, OPT_SCALE_KIND, OPT_SEED_LO, OPT_SEED_HI, OPT_FUSE_MODE, OPT_RIDGE, OPT_QUOT_EPS,
 OPT_TIMING, OPT_HOST_STAGING, OPT_REF_EVERY, OPT_COORD_OFFSET) = range(12)
(OK, ERR_INVALID_ARG, ERR_STATE, ERR_ALLOC, ERR_CUDA, ERR_NONFINITE, ERR_UNSUPPORTED) = range(7)
MAX_HISTORY = 16
TILE = 128

# every symbol include/tng.h declares
EXPORTS = [
    "tng_create", "tng_destroy", "tng_set_option", "tng_workspace_bytes", "tng_bind_workspace",
    "tng_push_reference", "tng_step", "tng_step_host", "tng_step_host_async", "tng_host_wait", "tng_fuse", "tng_encode", "tng_decode_aggregate",
    "tng_wire", "tng_wire_means", "tng_reference", "tng_history", "tng_stats", "tng_status_string", "tng_last_cuda_error",
    "tng_logistic_scratch_floats", "tng_logistic_grad", "tng_logistic_loss", "tng_rosenbrock_grad",
    "tng_rosenbrock_value", "tng_sgd_update", "tng_gram_static", "tng_state_bytes", "tng_save_state", "tng_load_state",
    "tng_selftest_bounded_wait", "tng_fuse_local", "tng_local_stats", "tng_local_stats_all", "tng_fuse_finish", "tng_encode_local", "tng_decode_commit",
    "tng_code_stride", "tng_quant8_rows", "tng_quant8_cols_scratch_bytes", "tng_quant8_cols", "tng_product8", "tng_linear8_scratch_bytes",
    "tng_linear8", "tng_linear8_grad_scratch_bytes", "tng_linear8_grad", "tng_dropout",
    "tng_embed", "tng_embed_grad_scratch_bytes", "tng_embed_grad", "tng_rmsnorm", "tng_rmsnorm_grad_scratch_bytes", "tng_rmsnorm_grad",
    "tng_orthogonalize_scratch_bytes", "tng_orthogonalize",
]


class Stats(C.Structure):
    _fields_ = [
        ("d", C.c_uint64), ("M", C.c_uint32), ("K", C.c_uint32), ("k", C.c_uint32), ("fuse_mode", C.c_uint32),
        ("rounds", C.c_uint64), ("bits_per_coord", C.c_double),
        ("alpha", C.c_double * MAX_HISTORY), ("gram", C.c_double * (MAX_HISTORY * MAX_HISTORY)),
        ("rhs", C.c_double * MAX_HISTORY), ("grad_sq", C.c_double), ("cnz", C.c_double),
        ("solver_fallback", C.c_uint32), ("pipeline_error", C.c_uint32),
        ("nonfinite_scales", C.c_uint64), ("kernel_launches", C.c_uint64), ("timed_rounds", C.c_uint64),
        ("ms_dots", C.c_double), ("ms_solve", C.c_double), ("ms_combine", C.c_double),
        ("ms_encode", C.c_double), ("ms_decode", C.c_double),
    ]


class Draw(C.Structure):
    """tng_draw: where an operator's random numbers come from (seed, layer, step, first row)."""
    _fields_ = [("seed_lo", C.c_uint32), ("seed_hi", C.c_uint32), ("layer", C.c_uint32), ("step", C.c_uint32),
                ("row0", C.c_uint64)]

    def __init__(self, seed=0, layer=0, step=0, row0=0):
        if not (0 <= seed < 1 << 64 and 0 <= layer < 1 << 30 and 0 <= step < 1 << 32 and 0 <= row0 <= 1 << 32):
            raise ValueError("seed, layer, step and row0 are unsigned of 64, 30, 32 and 32 bits")
        super().__init__(seed & 0xFFFFFFFF, seed >> 32, layer, step, row0)


class TngError(RuntimeError):
    def __init__(self, status, what):
        self.status = status
        super().__init__(f"{what}: {status_string(status)} (status {status})")


_lib = None


def lib():
    """Load libtng.so; there is no fallback if it has not been built."""
    global _lib
    if _lib is None:
        if not LIB_PATH.exists():
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_1901_08227_b200.build`")
        L = C.CDLL(str(LIB_PATH))
        vp, u64, u32, f32, f64 = C.c_void_p, C.c_uint64, C.c_uint32, C.c_float, C.c_double
        L.tng_create.argtypes = [C.POINTER(vp), u64, u32, u32, C.c_int, C.c_int]
        L.tng_destroy.argtypes = [vp]
        L.tng_destroy.restype = None
        L.tng_set_option.argtypes = [vp, C.c_int, f64]
        L.tng_workspace_bytes.argtypes = [vp, C.POINTER(C.c_size_t)]
        L.tng_bind_workspace.argtypes = [vp, vp, C.c_size_t]
        L.tng_push_reference.argtypes = [vp, vp, vp]
        L.tng_step.argtypes = [vp, vp, u64, vp, vp]
        L.tng_step_host.argtypes = [vp, vp, u64, vp, vp]
        L.tng_step_host_async.argtypes = [vp, vp, u64, vp, vp]
        L.tng_host_wait.argtypes = [vp]
        L.tng_fuse.argtypes = [vp, vp, u64, vp]
        L.tng_encode.argtypes = [vp, vp, u64, vp, u32, vp]
        L.tng_decode_aggregate.argtypes = [vp, vp, vp, vp]
        L.tng_wire.argtypes = [vp, C.POINTER(vp), C.POINTER(C.c_size_t), C.POINTER(vp), C.POINTER(C.c_size_t)]
        L.tng_wire_means.argtypes = [vp, C.POINTER(vp)]
        L.tng_reference.argtypes = [vp, C.POINTER(vp)]
        L.tng_history.argtypes = [vp, u32, C.POINTER(vp)]
        L.tng_stats.argtypes = [vp, C.POINTER(Stats)]
        L.tng_status_string.argtypes = [C.c_int]
        L.tng_status_string.restype = C.c_char_p
        L.tng_last_cuda_error.argtypes = [vp]
        L.tng_logistic_scratch_floats.argtypes = [u64, u64]
        L.tng_logistic_scratch_floats.restype = C.c_size_t
        L.tng_logistic_grad.argtypes = [vp, vp, u64, u64, vp, f32, vp, vp, vp]
        L.tng_logistic_loss.argtypes = [vp, vp, u64, u64, vp, f32, vp, vp, vp]
        L.tng_rosenbrock_grad.argtypes = [vp, u64, vp, u32, u64, vp, vp]
        L.tng_rosenbrock_value.argtypes = [vp, u64, vp, vp]
        L.tng_sgd_update.argtypes = [vp, vp, u64, f32, vp]
        L.tng_state_bytes.argtypes = [vp, C.POINTER(C.c_size_t)]
        L.tng_save_state.argtypes = [vp, vp, C.c_size_t, C.POINTER(C.c_size_t), vp]
        L.tng_load_state.argtypes = [vp, vp, C.c_size_t, vp]
        L.tng_fuse_local.argtypes = [vp, vp, u64, u32, vp]
        L.tng_local_stats.argtypes = [vp, C.POINTER(vp), C.POINTER(C.c_size_t)]
        L.tng_local_stats_all.argtypes = [vp, C.POINTER(vp), C.POINTER(C.c_size_t)]
        L.tng_selftest_bounded_wait.argtypes = [vp, C.POINTER(C.c_uint32), vp]
        L.tng_fuse_finish.argtypes = [vp, vp]
        L.tng_encode_local.argtypes = [vp, vp, u64, u32, u32, u32, vp]
        L.tng_decode_commit.argtypes = [vp, vp, vp]
        draw, st = C.POINTER(Draw), C.c_size_t
        L.tng_code_stride.argtypes, L.tng_code_stride.restype = [u64], st
        L.tng_quant8_rows.argtypes = [vp, C.c_int, u64, u64, u64, draw, vp, u64, vp, vp]
        L.tng_quant8_cols_scratch_bytes.argtypes, L.tng_quant8_cols_scratch_bytes.restype = [u64, u64], st
        L.tng_quant8_cols.argtypes = [vp, C.c_int, u64, u64, u64, draw, vp, u64, vp, vp, vp, vp]
        L.tng_product8.argtypes = [vp, u64, vp, vp, u64, vp, vp, u64, u64, u64, vp, C.c_int, u64, vp]
        L.tng_linear8_scratch_bytes.argtypes, L.tng_linear8_scratch_bytes.restype = [u64, u64], st
        L.tng_linear8.argtypes = [vp, C.c_int, u64, u64, u64, vp, u64, vp, u64, vp, vp, u64, vp, vp]
        L.tng_linear8_grad_scratch_bytes.argtypes, L.tng_linear8_grad_scratch_bytes.restype = [u64, u64, u64], st
        L.tng_linear8_grad.argtypes = [vp, u64, vp, u64, C.c_int, u64, u64, u64, vp, u64, vp, draw, vp, u64, vp, u64, vp, vp, vp]
        L.tng_dropout.argtypes = [vp, C.c_int, u64, u64, u64, vp, u64, f32, draw, vp, u64, vp]
        L.tng_embed.argtypes = [vp, C.c_int, u64, u64, u64, vp, u32, u64, f32, vp, C.c_int, u64, vp]
        L.tng_embed_grad_scratch_bytes.argtypes, L.tng_embed_grad_scratch_bytes.restype = [u64, u64], st
        L.tng_embed_grad.argtypes = [vp, C.c_int, u64, u64, u64, vp, u32, u64, f32, vp, u64, vp, vp]
        L.tng_rmsnorm.argtypes = [vp, C.c_int, u64, u64, u64, vp, u64, vp, f32, vp, u64, vp, u64, vp, u64, vp, vp, vp]
        L.tng_rmsnorm_grad_scratch_bytes.argtypes, L.tng_rmsnorm_grad_scratch_bytes.restype = [u64, u64], st
        L.tng_rmsnorm_grad.argtypes = [vp, u64, vp, u64, C.c_int, u64, u64, vp, vp, vp, u64, vp, u64, vp, vp, vp]
        L.tng_orthogonalize_scratch_bytes.argtypes, L.tng_orthogonalize_scratch_bytes.restype = [u64, u64, u64], st
        L.tng_orthogonalize.argtypes = [vp, C.c_int, u64, u64, u64, u64, u64, u32, f32, f32, f32, vp, C.c_int, u64, u64, vp, vp]
        L.tng_gram_static.argtypes = [C.POINTER(vp), u32, u64, vp, u32, u64, vp, vp]
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().tng_status_string(int(status)).decode()


def _check(status, what):
    if status != OK:
        raise TngError(status, what)


def _device(t=None) -> int:
    """The current device.  A CUDA tensor at hand says that CUDA is up, and the public call's checks (0.3 us) can be left out."""
    return torch._C._cuda_getDevice() if t is not None and t.is_cuda else torch.cuda.current_device()


def _stream(dev=None) -> int:
    """Handle of the current stream (of device `dev`).  current_stream() builds an object, 3 us a call: it serves where torch lacks
    the direct call."""
    dev = _device() if dev is None else dev
    try:
        return torch._C._cuda_getCurrentRawStream(dev)
    except AttributeError:
        return torch.cuda.current_stream(dev).cuda_stream


def _dev(t, dtype=torch.float32):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor):
        return int(t)                                  # a raw device address
    if not t.is_cuda or t.dtype != dtype:
        raise TypeError(f"expected a CUDA {dtype} tensor")
    return t.data_ptr()


def _rows(grads):
    """(M, d) CUDA float tensor with unit column stride -> (pointer, ld)."""
    if not grads.is_cuda or grads.dtype != torch.float32 or grads.dim() != 2 or grads.stride(1) != 1:
        raise TypeError("grads must be an (M, d) CUDA float32 tensor with contiguous rows")
    return grads.data_ptr(), grads.stride(0)


class Context:
    """One TNG reducer: d coordinates, M simulated workers, a ring of K past aggregates."""

    _OPTS = {"block": OPT_BLOCK, "qsgd_levels": OPT_QSGD_LEVELS, "scale_kind": OPT_SCALE_KIND,
             "seed_lo": OPT_SEED_LO, "seed_hi": OPT_SEED_HI, "fuse_mode": OPT_FUSE_MODE, "ridge": OPT_RIDGE,
             "quot_eps": OPT_QUOT_EPS, "timing": OPT_TIMING, "host_staging": OPT_HOST_STAGING, "ref_every": OPT_REF_EVERY,
             "coord_offset": OPT_COORD_OFFSET}

    def __init__(self, d, M, K, codec, norm, workspace=None, **options):
        self.d, self.M, self.K, self.codec, self.norm = int(d), int(M), int(K), int(codec), int(norm)
        h = C.c_void_p()
        _check(lib().tng_create(C.byref(h), self.d, self.M, self.K, self.codec, self.norm), "tng_create")
        self._h = h
        for key, val in options.items():
            self.set_option(key, val)
        self._ws = None
        if workspace is not None:
            self.bind_workspace(workspace)

    # -- lifetime
    def close(self):
        if getattr(self, "_h", None):
            lib().tng_destroy(self._h)
            self._h = None
            self._ws = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def set_option(self, key, value):
        key = self._OPTS[key] if isinstance(key, str) else int(key)
        _check(lib().tng_set_option(self._h, key, float(value)), "tng_set_option")

    def workspace_bytes(self) -> int:
        n = C.c_size_t()
        _check(lib().tng_workspace_bytes(self._h, C.byref(n)), "tng_workspace_bytes")
        return n.value

    def bind_workspace(self, buf: torch.Tensor):
        if not buf.is_cuda or not buf.is_contiguous():
            raise TypeError("workspace must be a contiguous CUDA tensor")
        _check(lib().tng_bind_workspace(self._h, buf.data_ptr(), buf.numel() * buf.element_size()), "tng_bind_workspace")
        self._ws = buf                                  # keep it alive

    # -- the round
    def push_reference(self, vec):
        _check(lib().tng_push_reference(self._h, _dev(vec), _stream()), "tng_push_reference")

    def step(self, grads, out=None):
        p, ld = _rows(grads)
        _check(lib().tng_step(self._h, p, ld, _dev(out), _stream()), "tng_step")
        return out

    def step_host(self, grads_host: torch.Tensor, out_host: torch.Tensor):
        if grads_host.is_cuda or out_host.is_cuda or grads_host.dtype != torch.float32 or grads_host.stride(1) != 1:
            raise TypeError("step_host takes host float32 tensors")
        _check(lib().tng_step_host(self._h, grads_host.data_ptr(), grads_host.stride(0), out_host.data_ptr(), _stream()),
               "tng_step_host")
        return out_host

    def step_host_async(self, grads_host: torch.Tensor, out_host: torch.Tensor):
        """step_host without waiting: out_host holds the aggregate after host_wait()."""
        if grads_host.is_cuda or out_host.is_cuda or grads_host.dtype != torch.float32 or grads_host.stride(1) != 1:
            raise TypeError("step_host_async takes host float32 tensors")
        _check(lib().tng_step_host_async(self._h, grads_host.data_ptr(), grads_host.stride(0), out_host.data_ptr(), _stream()),
               "tng_step_host_async")
        return out_host

    def host_wait(self):
        _check(lib().tng_host_wait(self._h), "tng_host_wait")

    def state_bytes(self) -> int:
        n = C.c_size_t()
        _check(lib().tng_state_bytes(self._h, C.byref(n)), "tng_state_bytes")
        return n.value

    def save_state(self) -> torch.Tensor:
        """The context's state (ring, round counter, held reference) as a host byte tensor."""
        buf = torch.empty(self.state_bytes(), dtype=torch.uint8)
        used = C.c_size_t()
        _check(lib().tng_save_state(self._h, buf.data_ptr(), buf.numel(), C.byref(used), _stream()), "tng_save_state")
        return buf[: used.value].clone()

    def load_state(self, buf: torch.Tensor):
        if buf.is_cuda or buf.dtype != torch.uint8 or not buf.is_contiguous():
            raise TypeError("state must be a contiguous host uint8 tensor")
        _check(lib().tng_load_state(self._h, buf.data_ptr(), buf.numel(), _stream()), "tng_load_state")

    # -- rank-local stages (workers spread over several GPUs)
    def fuse_local(self, grads):
        p, ld = _rows(grads)
        _check(lib().tng_fuse_local(self._h, p, ld, grads.shape[0], _stream()), "tng_fuse_local")

    def local_stats(self) -> torch.Tensor:
        """Zero-copy float64 view of the block to all-reduce (sum) between fuse_local and fuse_finish."""
        p, n = C.c_void_p(), C.c_size_t()
        _check(lib().tng_local_stats(self._h, C.byref(p), C.byref(n)), "tng_local_stats")
        return _view(p.value, (n.value,), torch.float64)

    def selftest_bounded_wait(self) -> bool:
        """True when a wait on a barrier that nothing completes ended by its poll limit (as it must)."""
        out = C.c_uint32(0)
        _check(lib().tng_selftest_bounded_wait(self._h, C.byref(out), _stream()), "tng_selftest_bounded_wait")
        return out.value == 1

    def local_stats_all(self) -> torch.Tensor:
        """The same for ranks that hold slices of the coordinates: Gram, rhs and grad_sq (273 doubles)."""
        p, n = C.c_void_p(), C.c_size_t()
        _check(lib().tng_local_stats_all(self._h, C.byref(p), C.byref(n)), "tng_local_stats_all")
        return _view(p.value, (n.value,), torch.float64)

    def fuse_finish(self):
        _check(lib().tng_fuse_finish(self._h, _stream()), "tng_fuse_finish")

    def encode_local(self, grads, m_first, step):
        p, ld = _rows(grads)
        _check(lib().tng_encode_local(self._h, p, ld, int(m_first), grads.shape[0], int(step), _stream()), "tng_encode_local")

    def decode_commit(self, out=None):
        _check(lib().tng_decode_commit(self._h, _dev(out), _stream()), "tng_decode_commit")
        return out

    def wire_views(self):
        """Zero-copy views of the wire, (M, words) int32 codes and (M, scales) float32, for collectives."""
        cp, wpw, sp, spw = self.wire_pointers()
        return _view(cp, (self.M, wpw), torch.int32), _view(sp, (self.M, spw), torch.float32)

    def fuse(self, grads):
        p, ld = _rows(grads)
        _check(lib().tng_fuse(self._h, p, ld, _stream()), "tng_fuse")

    def encode(self, grads, ref=None, step=0):
        p, ld = _rows(grads)
        _check(lib().tng_encode(self._h, p, ld, _dev(ref), int(step), _stream()), "tng_encode")

    def decode_aggregate(self, out, ref=None):
        _check(lib().tng_decode_aggregate(self._h, _dev(ref), _dev(out), _stream()), "tng_decode_aggregate")
        return out

    # -- views (cloned into fresh tensors on the current stream, so they stay valid)
    def wire(self):
        cp, sp = C.c_void_p(), C.c_void_p()
        wpw, spw = C.c_size_t(), C.c_size_t()
        _check(lib().tng_wire(self._h, C.byref(cp), C.byref(wpw), C.byref(sp), C.byref(spw)), "tng_wire")
        codes = _view(cp.value, (self.M, wpw.value), torch.int32).clone()
        scales = _view(sp.value, (self.M, spw.value), torch.float32).clone()
        return codes, scales

    def wire_pointers(self):
        cp, sp = C.c_void_p(), C.c_void_p()
        wpw, spw = C.c_size_t(), C.c_size_t()
        _check(lib().tng_wire(self._h, C.byref(cp), C.byref(wpw), C.byref(sp), C.byref(spw)), "tng_wire")
        return cp.value, wpw.value, sp.value, spw.value

    def wire_means_view(self):
        """Zero-copy view of the M scalar references (NORM_MEAN), for collectives."""
        p = C.c_void_p()
        _check(lib().tng_wire_means(self._h, C.byref(p)), "tng_wire_means")
        return _view(p.value, (self.M,), torch.float32)

    def wire_means(self):
        return self.wire_means_view().clone()

    def reference(self):
        p = C.c_void_p()
        _check(lib().tng_reference(self._h, C.byref(p)), "tng_reference")
        return _view(p.value, (self.d,), torch.float32).clone()

    def history(self, j):
        p = C.c_void_p()
        _check(lib().tng_history(self._h, int(j), C.byref(p)), "tng_history")
        return _view(p.value, (self.d,), torch.float32).clone()

    def stats(self, raise_on_nonfinite=False) -> Stats:
        s = Stats()
        st = lib().tng_stats(self._h, C.byref(s))
        if st != OK and not (st == ERR_NONFINITE and not raise_on_nonfinite):
            raise TngError(st, "tng_stats")
        return s

    def last_cuda_error(self) -> int:
        return lib().tng_last_cuda_error(self._h)


class _DeviceView:
    """Zero-copy view of library-owned device memory for torch (CUDA array interface)."""

    def __init__(self, ptr, shape, typestr):
        self.__cuda_array_interface__ = {"shape": tuple(shape), "typestr": typestr, "data": (int(ptr), False),
                                         "version": 2}


def _view(ptr, shape, dtype):
    typestr = {torch.float32: "<f4", torch.int32: "<i4", torch.float64: "<f8"}[dtype]
    return torch.as_tensor(_DeviceView(ptr, shape, typestr), device="cuda")


def gram_static(rows, grads, out):
    """tng_gram_static: Gram / rhs / mean squared norm of `rows` (list of (d,) CUDA tensors,
    newest first) against the (M, d) gradient rows, into `out` (k*k+k+1 float64 on the GPU).
    Allocates nothing on the device."""
    k = len(rows)
    arr = (C.c_void_p * max(k, 1))(*[_dev(r) for r in rows])
    p, ld = _rows(grads)
    d = rows[0].numel() if k else 0
    _check(lib().tng_gram_static(arr, k, d, p, grads.shape[0], ld, _dev(out, torch.float64), _stream()), "tng_gram_static")
    return out


# ---- producers -------------------------------------------------------------------------
def logistic_scratch_floats(n, d) -> int:
    return lib().tng_logistic_scratch_floats(int(n), int(d))


def logistic_grad(X, b, w, lambda2, grad, scratch):
    n, d = X.shape
    _check(lib().tng_logistic_grad(_dev(X), _dev(b), n, d, _dev(w), float(lambda2), _dev(grad), _dev(scratch), _stream()),
           "tng_logistic_grad")
    return grad


def logistic_loss(X, b, w, lambda2, loss, scratch):
    n, d = X.shape
    _check(lib().tng_logistic_loss(_dev(X), _dev(b), n, d, _dev(w), float(lambda2), _dev(loss, torch.float64),
                                   _dev(scratch), _stream()), "tng_logistic_loss")
    return loss


def rosenbrock_grad(x, noise, grads):
    p, ld = _rows(grads)
    if noise is not None:
        pn, ldn = _rows(noise)
        if ldn != ld:
            raise ValueError("noise and grads must share the row stride")
    else:
        pn = None
    _check(lib().tng_rosenbrock_grad(_dev(x), x.numel(), pn, grads.shape[0], ld, p, _stream()), "tng_rosenbrock_grad")
    return grads


def rosenbrock_value(x, value):
    _check(lib().tng_rosenbrock_value(_dev(x), x.numel(), _dev(value, torch.float64), _stream()), "tng_rosenbrock_value")
    return value


def sgd_update(w, v, eta):
    _check(lib().tng_sgd_update(_dev(w), _dev(v), w.numel(), float(eta), _stream()), "tng_sgd_update")
    return w


# ---- training-layer operators ------------------------------------------------------------
F32, BF16, F16 = 0, 1, 2
_DTYPE = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}


def _matrix(t, name, dtype=None, shape=None, dev=None):
    """A 2-D CUDA tensor of the current device (dev) with unit column stride -> (pointer, row stride)."""
    if t.get_device() != (_device() if dev is None else dev) or (t.dtype not in _DTYPE if dtype is None else t.dtype != dtype):
        raise TypeError(f"{name} must be a tensor on the current CUDA device of type {dtype or 'float32, bfloat16 or float16'}")
    size = t.shape
    if len(size) != 2 or (shape is not None and size != shape):
        raise ValueError(f"{name} has shape {tuple(size)}, expected {'two dimensions' if shape is None else tuple(shape)}")
    ld, unit = t.stride()
    rows, cols = size
    if unit != 1 and cols > 1:
        raise ValueError(f"{name} must have contiguous rows")
    return t.data_ptr(), ld if rows > 1 or ld > cols else cols


def _codes(t, name, shape=None, dev=None):
    """Codes to be read.  (What follows a line's end may be read up to the next multiple of 16, never used.)"""
    p, ld = _matrix(t, name, torch.int8, shape, dev)
    return p, ld if ld % 16 == 0 or t.shape[0] > 1 else -(-ld // 16) * 16


def _codes_out(t, name, shape):
    """Codes to be written, with zeros from each line's end to the next multiple of 16: the tensor has to own those bytes."""
    p, ld = _matrix(t, name, torch.int8, shape)
    lines, n = shape
    if lines and n and (lines == 1 and ld % 16 != 0 or
                        t.storage_offset() + (lines - 1) * ld + -(-n // 16) * 16 > t.untyped_storage().nbytes()):
        raise ValueError(f"{name} must hold every line up to the next multiple of 16 bytes (see empty_codes)")
    return p, ld


def _vector(t, name, n, dev=None):
    if t is None:
        return None
    if t.dtype != torch.float32 or t.get_device() != (_device() if dev is None else dev) or t.shape != (n,) or (n > 1 and t.stride(0) != 1):
        raise TypeError(f"{name} must be a contiguous float32 vector of {n} elements on the current CUDA device")
    return t.data_ptr()


def _scratch(buf, nbytes, like):
    """(pointer, owner) of at least nbytes; the owner is to be kept until the call has been enqueued."""
    if nbytes == 0:
        return None, None
    if buf is None:
        buf = like.new_empty(nbytes, dtype=torch.uint8)
    elif not buf.is_cuda or not buf.is_contiguous() or buf.numel() * buf.element_size() < nbytes or buf.device != like.device:
        raise ValueError(f"scratch must be a contiguous CUDA tensor of at least {nbytes} bytes")
    return buf.data_ptr(), buf


# sizes only: worth remembering, since a call through ctypes costs as much as the rest of the checks
@functools.lru_cache(maxsize=4096)
def _linear8_scratch(tokens, k):
    return lib().tng_linear8_scratch_bytes(tokens, k)


@functools.lru_cache(maxsize=4096)
def _linear8_grad_scratch(tokens, k, n):
    return lib().tng_linear8_grad_scratch_bytes(tokens, k, n)


def empty_codes(lines, n, device="cuda"):
    """Uninitialised codes of `lines` lines of n values, each line on a 16-byte boundary."""
    return torch.empty((lines, -(-n // 16) * 16), dtype=torch.int8, device=device)[:, :n]


def quant8_rows(x, draw=None, q=None, scale=None):
    """Codes of x by row and a scale per row: (rows, cols) int8, (rows,) float32.  Given a `q`, zeros are written
    from the end of each of its lines to the next multiple of 16 bytes."""
    p, ld = _matrix(x, "x")
    rows, cols = x.shape
    q = empty_codes(rows, cols, x.device) if q is None else q
    scale = torch.empty(rows, dtype=torch.float32, device=x.device) if scale is None else scale
    pq, ldq = _codes_out(q, "q", (rows, cols))
    _check(lib().tng_quant8_rows(p, _DTYPE[x.dtype], rows, cols, ld, draw, pq, ldq, _vector(scale, "scale", rows), _stream()),
           "tng_quant8_rows")
    return q, scale


def quant8_cols(x, draw=None, q=None, scale=None, colsum=None, scratch=None):
    """Codes of x by column, transposed, and a scale per column: (cols, rows) int8, (cols,) float32.
    `colsum` (cols float32) receives the column sums of x.  A `q` is filled up as by `quant8_rows`."""
    p, ld = _matrix(x, "x")
    rows, cols = x.shape
    q = empty_codes(cols, rows, x.device) if q is None else q
    scale = torch.empty(cols, dtype=torch.float32, device=x.device) if scale is None else scale
    pq, ldq = _codes_out(q, "q", (cols, rows))
    ps, _keep = _scratch(scratch, lib().tng_quant8_cols_scratch_bytes(rows, cols), x)
    _check(lib().tng_quant8_cols(p, _DTYPE[x.dtype], rows, cols, ld, draw, pq, ldq, _vector(scale, "scale", cols),
                                 _vector(colsum, "colsum", cols), ps, _stream()), "tng_quant8_cols")
    return q, scale


def product8(a, sa, b, sb, bias=None, dtype=torch.bfloat16, out=None):
    """out[i, j] = sum_l a[i, l] b[j, l] * sa[i] * sb[j] + bias[j]; a (m, k) and b (n, k) int8 codes."""
    m, k = a.shape
    n = b.shape[0]
    pa, lda = _codes(a, "a")
    pb, ldb = _codes(b, "b", (n, k))
    if out is None:
        out = torch.empty((m, n), dtype=dtype, device=a.device)
    po, ldo = _matrix(out, "out", None, (m, n))
    _check(lib().tng_product8(pa, lda, _vector(sa, "sa", m), pb, ldb, _vector(sb, "sb", n), _vector(bias, "bias", n), m, n, k,
                              po, _DTYPE[out.dtype], ldo, _stream()), "tng_product8")
    return out


def linear8(x, w, sw, bias=None, out=None, scratch=None):
    """y = x W^T + bias with x (tokens, k) coded by token in the call and W held as codes (n, k) with a
    scale per output channel (`quant8_rows` of W).  y has x's type."""
    dev = _device(x)
    px, ldx = _matrix(x, "x", None, None, dev)
    tokens, k = x.shape
    n = w.shape[0]
    pw, ldw = _codes(w, "w", (n, k), dev)
    if out is None:
        out = x.new_empty((tokens, n))
        po, ldo = out.data_ptr(), n
    else:
        po, ldo = _matrix(out, "out", x.dtype, (tokens, n), dev)
    nbytes = _linear8_scratch(tokens, k)
    ps, _keep = _scratch(scratch, nbytes, x) if nbytes else (None, None)
    status = lib().tng_linear8(px, _DTYPE[x.dtype], tokens, k, ldx, pw, ldw, _vector(sw, "sw", n, dev), n, _vector(bias, "bias", n, dev), po, ldo,
                               ps, _stream(dev))
    if status:
        raise TngError(status, "tng_linear8")
    return out


def linear8_grad(dy, x, wt, swt, draw=None, dx=None, dw=None, db=None, scratch=None):
    """Gradients of y = x W^T + bias: (dx, dw, db) from dy (tokens, n) and x (tokens, k).  `wt` (k, n) and
    `swt` (k) hold W by column (`quant8_cols` of W); with `draw` dy is rounded stochastically.  `dw` may be a
    strided float32 view, such as a part of a worker's row of gradients."""
    dev = _device(dy)
    py, ldy = _matrix(dy, "dy", None, None, dev)
    tokens, n = dy.shape
    k = x.shape[1]
    px, ldx = _matrix(x, "x", dy.dtype, (tokens, k), dev)
    pw, ldw = _codes(wt, "wt", (k, n), dev)
    if dx is None:
        dx = dy.new_empty((tokens, k))
        pdx, lddx = dx.data_ptr(), k
    else:
        pdx, lddx = _matrix(dx, "dx", dy.dtype, (tokens, k), dev)
    if dw is None:
        dw = dy.new_empty((n, k), dtype=torch.float32)
        pdw, lddw = dw.data_ptr(), k
    else:
        pdw, lddw = _matrix(dw, "dw", torch.float32, (n, k), dev)
    if db is None:
        db = dy.new_empty(n, dtype=torch.float32)
        pdb = db.data_ptr()
    else:
        pdb = _vector(db, "db", n, dev)
    ps, _keep = _scratch(scratch, _linear8_grad_scratch(tokens, k, n), dy)
    _check(lib().tng_linear8_grad(py, ldy, px, ldx, _DTYPE[dy.dtype], tokens, k, n, pw, ldw, _vector(swt, "swt", k, dev), draw,
                                  pdx, lddx, pdw, lddw, pdb, ps, _stream(dev)), "tng_linear8_grad")
    return dx, dw, db


def dropout(x, p, draw, residual=None, out=None):
    """residual + dropout(x): kept elements are scaled by 1/(1-p); the mask follows from `draw` alone."""
    dev = _device(x)
    px, ldx = _matrix(x, "x", None, None, dev)
    rows, cols = x.shape
    if out is None:
        out = torch.empty_like(x)
        po, ldo = out.data_ptr(), cols if rows == 1 else out.stride(0)
    else:
        po, ldo = _matrix(out, "out", x.dtype, x.shape, dev)
    pr, ldr = (None, 0) if residual is None else _matrix(residual, "residual", x.dtype, x.shape, dev)
    status = lib().tng_dropout(px, _DTYPE[x.dtype], rows, cols, ldx, pr, ldr, p, draw, po, ldo, _stream(dev))
    if status:
        raise TngError(status, "tng_dropout")
    return out


def dropout_grad(dy, p, draw, out=None):
    """Gradient of `dropout` with respect to x (with respect to the residual it is dy itself)."""
    return dropout(dy, p, draw, None, out)


# ---- token models -------------------------------------------------------------------------
_ID_BYTES = {torch.int64: 8, torch.int32: 4}


def _ids(t, dev):
    """Token ids, one-dimensional and contiguous -> (pointer, bytes an id, how many)."""
    if t.get_device() != dev or t.dtype not in _ID_BYTES:
        raise TypeError("ids must be an int64 or int32 tensor on the current CUDA device")
    if t.dim() != 1 or (t.shape[0] > 1 and t.stride(0) != 1):
        raise ValueError("ids must be one-dimensional and contiguous")
    return t.data_ptr(), _ID_BYTES[t.dtype], t.shape[0]


@functools.lru_cache(maxsize=4096)
def _embed_grad_scratch(tokens, width):
    return lib().tng_embed_grad_scratch_bytes(tokens, width)


@functools.lru_cache(maxsize=4096)
def _rmsnorm_grad_scratch(rows, cols):
    return lib().tng_rmsnorm_grad_scratch_bytes(rows, cols)


def embed(table, ids, scale=1.0, dtype=None, out=None):
    """out[t] = table[ids[t]] * scale, in `dtype` (the table's unless given).  An id of -1 is an empty place (a row of zeros); any
    other id outside the table gives a row of NaN."""
    dev = _device(table)
    pt, ldt = _matrix(table, "table", None, None, dev)
    pi, id_bytes, tokens = _ids(ids, dev)
    vocab, width = table.shape
    if out is None:
        if dtype is not None and dtype not in _DTYPE:
            raise TypeError(f"dtype must be float32, bfloat16 or float16, not {dtype}")
        out = table.new_empty((tokens, width), dtype=table.dtype if dtype is None else dtype)
        po, ldo = out.data_ptr(), width
    else:
        if dtype is not None and out.dtype != dtype:
            raise TypeError(f"out is {out.dtype}, dtype says {dtype}")
        po, ldo = _matrix(out, "out", None, (tokens, width), dev)
    status = lib().tng_embed(pt, _DTYPE[table.dtype], vocab, width, ldt, pi, id_bytes, tokens, scale, po, _DTYPE[out.dtype], ldo, _stream(dev))
    if status:
        raise TngError(status, "tng_embed")
    return out


def embed_grad(dy, ids, vocab, scale=1.0, dtable=None, scratch=None):
    """Gradient of `embed` with respect to the table, (vocab, width) float32, every row written.  `dtable` may be a strided view,
    such as a part of a worker's row of gradients."""
    dev = _device(dy)
    py, ldy = _matrix(dy, "dy", None, None, dev)
    tokens, width = dy.shape
    pi, id_bytes, n = _ids(ids, dev)
    if n != tokens:
        raise ValueError(f"{n} ids for {tokens} rows of dy")
    dtable, pd, ldd = _made(dtable, "dtable", torch.float32, (vocab, width), dev, dy)
    ps, _keep = _scratch(scratch, _embed_grad_scratch(tokens, width), dy)
    status = lib().tng_embed_grad(py, _DTYPE[dy.dtype], tokens, width, ldy, pi, id_bytes, vocab, scale, pd, ldd, ps, _stream(dev))
    if status:
        raise TngError(status, "tng_embed_grad")
    return dtable


def _made(t, name, dtype, shape, dev, like):
    """An output (rows, cols) -> (tensor, pointer, row stride): the one given, checked, or a new one, which needs no check."""
    if t is None:
        t = like.new_empty(shape, dtype=dtype)
        return t, t.data_ptr(), shape[1]
    p, ld = _matrix(t, name, dtype, shape, dev)
    return t, p, ld


def _made_vector(t, name, n, dev, like):
    if t is None:
        t = like.new_empty(n, dtype=torch.float32)
        return t, t.data_ptr()
    return t, _vector(t, name, n, dev)


def _norm_inputs(x, w, residual, h):
    """What both norms do first -> (dev, dtype, shape, h, pointers and strides of x, residual, w and h)."""
    dev = _device(x)
    px, ldx = _matrix(x, "x", None, None, dev)
    dtype, shape = x.dtype, x.shape
    pw = _vector(w, "w", shape[1], dev)
    if pw is None:
        raise TypeError("w must be a contiguous float32 vector on the current CUDA device")
    if residual is None:
        pr, ldr = None, 0
        ph, ldh = (None, 0) if h is None else _matrix(h, "h", dtype, shape, dev)
    else:
        pr, ldr = _matrix(residual, "residual", dtype, shape, dev)
        h, ph, ldh = _made(h, "h", dtype, shape, dev, x)
    return dev, dtype, shape, h, (px, ldx, pr, ldr, pw, ph, ldh)


def rmsnorm(x, w, eps=1e-6, residual=None, h=None, y=None, r=None):
    """(y, h, r): h = x + residual (x itself without one), r = 1/sqrt(mean(h^2) + eps) by row, y = h r w in x's type.  w is float32.
    `h` may be x's or the residual's own tensor, `y` x's."""
    dev, dtype, shape, h, (px, ldx, pr, ldr, pw, ph, ldh) = _norm_inputs(x, w, residual, h)
    rows, cols = shape
    y, py, ldy = _made(y, "y", dtype, shape, dev, x)
    r, p_r = _made_vector(r, "r", rows, dev, x)
    status = lib().tng_rmsnorm(px, _DTYPE[dtype], rows, cols, ldx, pr, ldr, pw, eps, ph, ldh, py, ldy, None, 0, None, p_r, _stream(dev))
    if status:
        raise TngError(status, "tng_rmsnorm")
    return y, x if h is None else h, r


def rmsnorm8(x, w, eps=1e-6, residual=None, h=None, q=None, scale=None, r=None, y=None):
    """(q, scale, h, r): `rmsnorm` with its output as 8-bit codes by row and a scale per row, as `product8` takes them.  Given a `y`,
    the rows are written there in x's type too (what `linear8_grad` takes).  A `q` is filled up as by `quant8_rows`."""
    dev, dtype, shape, h, (px, ldx, pr, ldr, pw, ph, ldh) = _norm_inputs(x, w, residual, h)
    rows, cols = shape
    if q is None:
        ldq = -(-cols // 16) * 16
        q = x.new_empty((rows, ldq), dtype=torch.int8)
        pq = q.data_ptr()
        if ldq != cols:
            q = q[:, :cols]
    else:
        pq, ldq = _codes_out(q, "q", shape)
    py, ldy = (None, 0) if y is None else _matrix(y, "y", dtype, shape, dev)
    scale, ps = _made_vector(scale, "scale", rows, dev, x)
    r, p_r = _made_vector(r, "r", rows, dev, x)
    status = lib().tng_rmsnorm(px, _DTYPE[dtype], rows, cols, ldx, pr, ldr, pw, eps, ph, ldh, py, ldy, pq, ldq, ps, p_r, _stream(dev))
    if status:
        raise TngError(status, "tng_rmsnorm")
    return q, scale, x if h is None else h, r


def rmsnorm_grad(dy, h, w, r, dres=None, dx=None, dw=None, scratch=None):
    """(dx, dw) of `rmsnorm` and `rmsnorm8` from dy, the gradient of y, with the h and r that they returned.  dx is the gradient of
    x and of the residual alike; `dres` (what reaches h on its other ways) is added to it.  dx may be dy's or dres's own tensor."""
    dev = _device(dy)
    py, ldy = _matrix(dy, "dy", None, None, dev)
    shape, dtype = dy.shape, dy.dtype
    rows, cols = shape
    ph, ldh = _matrix(h, "h", dtype, shape, dev)
    pr, ldr = (None, 0) if dres is None else _matrix(dres, "dres", dtype, shape, dev)
    dx, px, ldx = _made(dx, "dx", dtype, shape, dev, dy)
    dw, pdw = _made_vector(dw, "dw", cols, dev, dy)
    ps, _keep = _scratch(scratch, _rmsnorm_grad_scratch(rows, cols), dy)
    status = lib().tng_rmsnorm_grad(py, ldy, ph, ldh, _DTYPE[dtype], rows, cols, _vector(w, "w", cols, dev), _vector(r, "r", rows, dev),
                                    pr, ldr, px, ldx, pdw, ps, _stream(dev))
    if status:
        raise TngError(status, "tng_rmsnorm_grad")
    return dx, dw


# ---- updates of weight matrices -------------------------------------------------------------
@functools.lru_cache(maxsize=4096)
def _orthogonalize_scratch(batch, rows, cols):
    return lib().tng_orthogonalize_scratch_bytes(batch, rows, cols)


def _matrices(t, name, shape, dev):
    """One matrix (rows, cols) or a batch (batch, rows, cols), each row contiguous -> (pointer, row stride, stride of the batch)."""
    if t.get_device() != dev or t.dtype not in _DTYPE:
        raise TypeError(f"{name} must be a tensor on the current CUDA device of type float32, bfloat16 or float16")
    if t.dim() not in (2, 3) or (shape is not None and t.shape != shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {'two or three dimensions' if shape is None else tuple(shape)}")
    rows, cols = t.shape[-2:]
    ld, unit = t.stride()[-2:]
    if unit != 1 and cols > 1:
        raise ValueError(f"{name} must have contiguous rows")
    return t.data_ptr(), ld if rows > 1 or ld > cols else cols, t.stride(0) if t.dim() == 3 else 0


def orthogonalize(v, steps=5, coefficients=(3.4445, -4.7750, 2.0315), dtype=None, out=None, scratch=None):
    """The orthogonalised update of a matrix (rows, cols), or of each of a batch: X = v / |v| and `steps` times
    X <- (a I + b G + c G^2) X with G = X X^T, which brings all singular values near one.  `v` may be a view of the aggregate that
    `Context.step` returns; the result has v's type unless `dtype` or `out` says otherwise.  Rows or columns of less than 1e-4 of the largest
    ones' norm keep fewer than fp32's digits (about 4e-10 over that fraction is their relative error)."""
    dev = _device(v)
    pv, ldv, stride = _matrices(v, "v", None, dev)
    batch, (rows, cols) = v.shape[0] if v.dim() == 3 else 1, v.shape[-2:]
    a, b, c = coefficients
    if out is None:
        out = v.new_empty(v.shape, dtype=v.dtype if dtype is None else dtype)
    elif dtype is not None and out.dtype != dtype:
        raise TypeError(f"out is {out.dtype}, dtype says {dtype}")
    po, ldo, out_stride = _matrices(out, "out", v.shape, dev)
    ps, _keep = _scratch(scratch, _orthogonalize_scratch(batch, rows, cols), v)
    status = lib().tng_orthogonalize(pv, _DTYPE[v.dtype], batch, rows, cols, ldv, stride, steps, a, b, c, po, _DTYPE[out.dtype], ldo, out_stride,
                                     ps, _stream(dev))
    if status:
        raise TngError(status, "tng_orthogonalize")
    return out
