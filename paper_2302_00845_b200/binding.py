"""ctypes binding of libcdgrab.so: same names as ``include/cdgrab.h``, argument marshalling only.

Every step of the path runs in the library's CUDA kernels.  There is no CPU fallback: if the
shared library has not been built, or no sm_100 device is present, the calls raise.
PyTorch tensors are used as device buffers; their ``data_ptr()`` and the current CUDA stream
handle are what crosses the boundary.
"""
from __future__ import annotations

import ctypes as C
import os
import struct

HERE = os.path.dirname(os.path.abspath(__file__))
# CDGRAB_LIB: file name (inside the package) of a diagnostic build to load instead
LIB_PATH = os.path.join(HERE, os.path.basename(os.environ.get("CDGRAB_LIB", "libcdgrab.so")))

F32, BF16 = 0, 1
OK = 0
ERR_INVALID, ERR_STATE, ERR_CUDA, ERR_NOMEM, ERR_NONFINITE, ERR_TIMEOUT, ERR_DEVICE = -1, -2, -3, -4, -5, -6, -7
ERR_TOO_LARGE = -8
ERR_CORRUPT = -9
PATH_AUTO, PATH_FUSED, PATH_FMA, PATH_UMMA = 0, 1, 2, 3
KERNEL_KINDS = ("gram", "combine", "scan", "update", "fused", "logreg")
PATH_NAMES = {PATH_FUSED: "fused", PATH_FMA: "fma", PATH_UMMA: "umma", 4: "independent", 5: "literal"}


class AttentionShape(C.Structure):
    """cdgrab_attention_shape: sizes, and strides in elements for (batch, token, head)."""
    _fields_ = [(n, C.c_int) for n in ("batch", "len_q", "len_kv", "heads", "kv_heads", "head_dim", "causal")] + \
               [("scale", C.c_float)] + \
               [(n + "_stride", C.c_longlong * 3) for n in ("q", "k", "v", "o", "do", "dq", "dk", "dv")]


# name -> (restype, argtypes); the single list of what include/cdgrab.h declares
SIGNATURES = {
    "cdgrab_create": (C.c_int, [C.c_int, C.c_int, C.c_longlong, C.c_int, C.POINTER(C.c_void_p)]),
    "cdgrab_create_independent": (C.c_int, [C.c_int, C.c_int, C.c_longlong, C.c_int, C.POINTER(C.c_void_p)]),
    "cdgrab_get_r_worker": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p]),
    "cdgrab_create_shard": (C.c_int, [C.c_int, C.c_int, C.c_longlong, C.c_int, C.POINTER(C.c_void_p)]),
    "cdgrab_step_begin": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "cdgrab_step_finish": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "cdgrab_destroy": (C.c_int, [C.c_void_p]),
    "cdgrab_set_perms": (C.c_int, [C.c_void_p, C.c_void_p]),
    "cdgrab_begin_epoch": (C.c_int, [C.c_void_p, C.c_void_p]),
    "cdgrab_step": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p]),
    "cdgrab_step_randomized": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_double, C.c_void_p]),
    "cdgrab_out_of_bound": (C.c_longlong, [C.c_void_p]),
    "cdgrab_step_randomized_seeded": (C.c_int, [C.c_void_p, C.c_void_p, C.c_ulonglong, C.c_uint, C.c_double, C.c_void_p]),
    "cdgrab_randomized_uniforms": (C.c_int, [C.c_ulonglong, C.c_uint, C.c_uint, C.c_int, C.c_void_p, C.c_void_p]),
    "cdgrab_step_mean": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "cdgrab_end_epoch": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p]),
    "cdgrab_get_signs": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p]),
    "cdgrab_get_r": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p]),
    "cdgrab_get_margins": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p]),
    "cdgrab_get_perms": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p]),
    "cdgrab_get_next_perms": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p]),
    "cdgrab_status": (C.c_int, [C.c_void_p]),
    "cdgrab_clear_status": (C.c_int, [C.c_void_p]),
    "cdgrab_selftest_wait_timeout": (C.c_int, [C.c_void_p, C.c_longlong, C.POINTER(C.c_longlong)]),
    "cdgrab_state_bytes": (C.c_longlong, [C.c_void_p]),
    "cdgrab_save_state": (C.c_int, [C.c_void_p, C.c_void_p, C.c_longlong]),
    "cdgrab_load_state": (C.c_int, [C.c_void_p, C.c_void_p, C.c_longlong]),
    "cdgrab_path": (C.c_int, [C.c_void_p]),
    "cdgrab_launch_count": (C.c_longlong, [C.c_void_p]),
    "cdgrab_strerror": (C.c_char_p, [C.c_int]),
    "cdgrab_step_many": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int, C.c_void_p]),
    "cdgrab_profile_enable": (C.c_int, [C.c_void_p, C.c_int]),
    "cdgrab_profile_read": (C.c_int, [C.c_void_p, C.c_int, C.POINTER(C.c_double), C.POINTER(C.c_longlong)]),
    "cdgrab_logreg_grads": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "cdgrab_step_logreg": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "cdgrab_step_host": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "cdgrab_herding_workspace_bytes": (C.c_longlong, [C.c_int, C.c_int, C.c_longlong]),
    "cdgrab_herding_objective": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_longlong, C.c_void_p,
                                           C.c_longlong, C.c_void_p, C.c_void_p]),
    "cdgrab_step_noalloc": (C.c_int, [C.c_int, C.c_longlong, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p,
                                      C.c_void_p]),
    "cdgrab_noalloc_status": (C.c_int, []),
    "cdgrab_layer_norm_forward": (C.c_int, [C.c_longlong, C.c_int, C.c_int, C.c_void_p, C.c_longlong, C.c_void_p,
                                            C.c_void_p, C.c_float, C.c_void_p, C.c_longlong, C.c_void_p, C.c_void_p,
                                            C.c_void_p]),
    "cdgrab_layer_norm_workspace_bytes": (C.c_longlong, [C.c_int, C.c_longlong, C.c_int]),
    "cdgrab_layer_norm_backward": (C.c_int, [C.c_int, C.c_longlong, C.c_int, C.c_int, C.c_void_p, C.c_longlong,
                                             C.c_void_p, C.c_longlong, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                             C.c_longlong, C.c_int, C.c_void_p, C.c_void_p, C.c_longlong, C.c_void_p,
                                             C.c_longlong, C.c_void_p]),
    "cdgrab_attention_forward": (C.c_int, [C.POINTER(AttentionShape)] + [C.c_void_p] * 8),
    "cdgrab_attention_workspace_bytes": (C.c_longlong, [C.POINTER(AttentionShape)]),
    "cdgrab_attention_backward": (C.c_int, [C.POINTER(AttentionShape)] + [C.c_void_p] * 12 + [C.c_longlong, C.c_void_p]),
    "cdgrab_orthogonalise_workspace_bytes": (C.c_longlong, [C.c_int, C.c_int, C.c_int]),
    "cdgrab_orthogonalise": (C.c_int, [C.c_int, C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_longlong, C.c_longlong,
                                       C.c_int, C.POINTER(C.c_float), C.c_float, C.c_void_p, C.c_longlong,
                                       C.c_longlong, C.c_void_p, C.c_longlong, C.c_void_p]),
    "cdgrab_operators_status": (C.c_int, []),
    "cdgrab_operators_wait_limit": (C.c_int, [C.c_longlong]),
}

_lib = None


class CdgrabError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        msg = lib().cdgrab_strerror(code).decode() if _lib is not None else str(code)
        super().__init__(f"{where}: {msg} ({code})")


def lib() -> C.CDLL:
    """Load libcdgrab.so (built in-tree by ``paper_2302_00845_b200.build``); raises if absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2302_00845_b200.build` "
                "(there is no CPU fallback)")
        l = C.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(l, name)
            fn.restype = res
            fn.argtypes = args
        _lib = l
    return _lib


def _check(code: int, where: str):
    if code != OK:
        raise CdgrabError(code, where)


def _stream_ptr(stream=None):
    import torch
    s = stream if stream is not None else torch.cuda.current_stream()
    return C.c_void_p(s.cuda_stream)


def _ptr(t):
    """Raw pointer of a contiguous torch tensor or numpy array."""
    if hasattr(t, "data_ptr"):
        assert t.is_contiguous()
        return C.c_void_p(t.data_ptr())
    assert t.flags["C_CONTIGUOUS"]
    return C.c_void_p(t.ctypes.data)


class CdGrab:
    """Order-server state for m workers x n items in R^d (see ``include/cdgrab.h``)."""

    def __init__(self, m: int, n: int, d: int, dtype: str | int = "f32", independent: bool = False,
                 shard: bool = False):
        code = {"f32": F32, "bf16": BF16}.get(dtype, dtype)
        h = C.c_void_p()
        if shard:         # one column shard of a coordinated order: d is the shard's width
            _check(lib().cdgrab_create_shard(m, n, d, code, C.byref(h)), "cdgrab_create_shard")
        elif independent:   # ID-GraB (PairBal): one running sum per worker
            _check(lib().cdgrab_create_independent(m, n, d, code, C.byref(h)), "cdgrab_create_independent")
        else:
            _check(lib().cdgrab_create(m, n, d, code, C.byref(h)), "cdgrab_create")
        self._h = h
        self.m, self.n, self.d, self.dtype = m, n, d, code

    # life cycle -------------------------------------------------------------------------
    def destroy(self):
        if getattr(self, "_h", None):
            lib().cdgrab_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.destroy()

    # the calls of the header ----------------------------------------------------------------
    def set_perms(self, perms):
        _check(lib().cdgrab_set_perms(self._h, _ptr(perms)), "cdgrab_set_perms")

    def begin_epoch(self, stream=None):
        _check(lib().cdgrab_begin_epoch(self._h, _stream_ptr(stream)), "cdgrab_begin_epoch")

    def step(self, grads, stream=None):
        """grads: CUDA tensor [2][m][d] of the handle's dtype."""
        _check(lib().cdgrab_step(self._h, _ptr(grads), _stream_ptr(stream)), "cdgrab_step")

    def step_randomized(self, grads, u, w: float, stream=None):
        """step() under the randomized rule: u CUDA float32 [m] uniforms, w > 0 the bound."""
        _check(lib().cdgrab_step_randomized(self._h, _ptr(grads), _ptr(u), float(w), _stream_ptr(stream)),
               "cdgrab_step_randomized")

    def step_randomized_seeded(self, grads, seed: int, epoch: int, w: float, stream=None):
        """step() under the randomized rule with the library's own counter-based draws."""
        _check(lib().cdgrab_step_randomized_seeded(self._h, _ptr(grads), int(seed), int(epoch), float(w),
                                                   _stream_ptr(stream)), "cdgrab_step_randomized_seeded")

    @property
    def out_of_bound(self) -> int:
        return int(lib().cdgrab_out_of_bound(self._h))

    def step_begin(self, grads, gram_out, stream=None):
        """Shard handle: pass 1; gram_out is a CUDA float64 tensor [m*m + m] for the partial (G, b)."""
        _check(lib().cdgrab_step_begin(self._h, _ptr(grads), _ptr(gram_out), _stream_ptr(stream)),
               "cdgrab_step_begin")

    def step_finish(self, grads, gram_in, stream=None):
        """Shard handle: decisions on the summed (G, b) and the update of this shard's slice of r."""
        _check(lib().cdgrab_step_finish(self._h, _ptr(grads), _ptr(gram_in), _stream_ptr(stream)),
               "cdgrab_step_finish")

    def step_mean(self, grads, mean_out, stream=None):
        """step() that also writes the average of each gather buffer into mean_out (CUDA float32 [2][d])."""
        _check(lib().cdgrab_step_mean(self._h, _ptr(grads), _ptr(mean_out), _stream_ptr(stream)),
               "cdgrab_step_mean")

    def step_many(self, grads, stream=None):
        """grads: contiguous CUDA tensor [count][2][m][d]; the count steps in one call."""
        _check(lib().cdgrab_step_many(self._h, _ptr(grads), int(grads.shape[0]), _stream_ptr(stream)),
               "cdgrab_step_many")

    def step_logreg(self, X, y, w, stream=None):
        """One balancing step straight from the feature rows (no gradient buffer)."""
        _check(lib().cdgrab_step_logreg(self._h, _ptr(X), _ptr(y), _ptr(w), _stream_ptr(stream)),
               "cdgrab_step_logreg")

    def step_host(self, grads_host, staging, stream=None):
        """grads_host: pinned host tensor [2][m][d]; staging: CUDA tensor of the same size."""
        _check(lib().cdgrab_step_host(self._h, _ptr(grads_host), _ptr(staging), _stream_ptr(stream)),
               "cdgrab_step_host")

    def end_epoch(self, perms_out=None, stream=None):
        p = _ptr(perms_out) if perms_out is not None else None
        _check(lib().cdgrab_end_epoch(self._h, p, _stream_ptr(stream)), "cdgrab_end_epoch")

    def logreg_grads(self, X, y, w, grads_out, stream=None):
        _check(lib().cdgrab_logreg_grads(self._h, _ptr(X), _ptr(y), _ptr(w), _ptr(grads_out),
                                         _stream_ptr(stream)), "cdgrab_logreg_grads")

    # read-back ------------------------------------------------------------------------------
    def _fetch(self, name, shape, dtype):
        import torch
        out = torch.empty(shape, dtype=dtype, device="cuda")
        _check(getattr(lib(), name)(self._h, _ptr(out), _stream_ptr()), name)
        torch.cuda.current_stream().synchronize()
        return out

    def signs(self):
        import torch
        return self._fetch("cdgrab_get_signs", (self.m, self.n // 2), torch.int8)

    def r(self):
        import torch
        return self._fetch("cdgrab_get_r", (self.d,), torch.float32)

    def r_worker(self, i: int):
        import torch
        out = torch.empty(self.d, dtype=torch.float32, device="cuda")
        _check(lib().cdgrab_get_r_worker(self._h, i, _ptr(out), _stream_ptr()), "cdgrab_get_r_worker")
        torch.cuda.current_stream().synchronize()
        return out

    def margins(self):
        import torch
        return self._fetch("cdgrab_get_margins", (self.m, self.n // 2), torch.float32)

    def perms(self):
        import torch
        return self._fetch("cdgrab_get_perms", (self.m, self.n), torch.int32)

    def next_perms(self):
        import torch
        return self._fetch("cdgrab_get_next_perms", (self.m, self.n), torch.int32)

    def save_state(self):
        """Host copy (numpy uint8 array) of everything needed to continue in another handle."""
        import numpy as np
        nbytes = int(lib().cdgrab_state_bytes(self._h))
        buf = np.empty(nbytes, dtype=np.uint8)
        _check(lib().cdgrab_save_state(self._h, buf.ctypes.data, nbytes), "cdgrab_save_state")
        return buf

    def load_state(self, buf):
        _check(lib().cdgrab_load_state(self._h, buf.ctypes.data, int(buf.nbytes)), "cdgrab_load_state")

    def status(self) -> int:
        return lib().cdgrab_status(self._h)

    def check_status(self):
        _check(self.status(), "cdgrab_status")

    def profile_enable(self, on: bool = True):
        _check(lib().cdgrab_profile_enable(self._h, int(on)), "cdgrab_profile_enable")

    def profile_read(self) -> dict:
        """{kernel kind: (total ms, launches)} for the launches recorded since profiling was enabled."""
        out = {}
        for kind, name in enumerate(KERNEL_KINDS):
            ms, cnt = C.c_double(), C.c_longlong()
            _check(lib().cdgrab_profile_read(self._h, kind, C.byref(ms), C.byref(cnt)), "cdgrab_profile_read")
            if cnt.value:
                out[name] = (ms.value, cnt.value)
        return out

    @property
    def path(self) -> str:
        return PATH_NAMES.get(lib().cdgrab_path(self._h), "?")

    @property
    def launch_count(self) -> int:
        return int(lib().cdgrab_launch_count(self._h))


def step_noalloc(grads, r, signs_out, stream=None):
    """cdgrab_step_noalloc on torch tensors: grads [2][m][d] (f32 or bf16), r float32 [d] updated in
    place, signs_out int8 [m].  Allocates nothing on the device."""
    import torch
    m, d = int(grads.shape[1]), int(grads.shape[2])
    code = F32 if grads.dtype == torch.float32 else BF16
    _check(lib().cdgrab_step_noalloc(m, d, code, _ptr(grads), _ptr(r), _ptr(signs_out), _stream_ptr(stream)),
           "cdgrab_step_noalloc")


def randomized_uniforms(seed: int, epoch: int, k: int, m: int, stream=None):
    """The m draws of (seed, epoch, k) as a CUDA float32 tensor."""
    import torch
    out = torch.empty(m, dtype=torch.float32, device="cuda")
    _check(lib().cdgrab_randomized_uniforms(int(seed), int(epoch), int(k), m, _ptr(out), _stream_ptr(stream)),
           "cdgrab_randomized_uniforms")
    return out


def noalloc_status() -> int:
    """cdgrab_noalloc_status: the device status of the step_noalloc calls so far (read and cleared)."""
    return int(lib().cdgrab_noalloc_status())


def herding_objective(z, perms, stream=None) -> float:
    """Eq. (7) on the device: z CUDA float32 [m][n][d] (by item id), perms CUDA int32 [m][n]."""
    import torch
    m, n, d = (int(v) for v in z.shape)
    nbytes = int(lib().cdgrab_herding_workspace_bytes(m, n, d))
    ws = torch.empty(nbytes // 8, dtype=torch.float64, device=z.device)
    out = torch.empty(1, dtype=torch.float64, device=z.device)
    _check(lib().cdgrab_herding_objective(_ptr(z), _ptr(perms), m, n, d, _ptr(ws), nbytes, _ptr(out),
                                          _stream_ptr(stream)), "cdgrab_herding_objective")
    return float(out.item())


# ---- training operators --------------------------------------------------------------------------
# A call costs a few microseconds of host time, as much as a small operator takes on the device: checks
# build their messages only when they fail, and shapes cross the boundary as one packed struct.
# `stream`: the torch stream to run on, the current one by default.  The caller orders it after what makes the inputs;
# the tensors that are passed are kept from reuse until it has got past the call, and what is returned belongs to it, as
# under torch.cuda.stream.
torch = None          # imported by the first call: the module itself loads, and finds the library, without it
_SHAPE = struct.Struct("7if24q")          # cdgrab_attention_shape
_INT_MAX = 2 ** 31 - 1                    # ctypes passes the low 32 bits of a larger number without a word


def _use_torch():
    global torch, _CODES, _raw_stream
    import torch as t
    _CODES = {t.float32: F32, t.bfloat16: BF16}
    _raw_stream = getattr(t._C, "_cuda_getCurrentRawStream", None) or (lambda dev: t.cuda.current_stream(dev).cuda_stream)
    torch = t             # last: it tells other threads that the rest is there


def _place(stream, *tensors):
    """Where an operator runs: the raw stream, and the torch stream whose pool its outputs and scratch come
    from when that is not the current one (so that freeing them is ordered after the launches).  The tensors, which
    come from other streams' pools then, are recorded on it."""
    if torch is None:
        _use_torch()
    dev = torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise ValueError("tensors have to be on the current CUDA device")
    current = _raw_stream(dev)
    if stream is None or stream.cuda_stream == current:
        return current, None
    for t in tensors:
        if t is not None:
            t.record_stream(stream)
    return stream.cuda_stream, stream


def _empty(like, shape, dtype, other):
    if other is None:       # (naming the type costs half a microsecond)
        return like.new_empty(shape) if like.dtype is dtype else like.new_empty(shape, dtype=dtype)
    with torch.cuda.stream(other):
        return like.new_empty(shape, dtype=dtype)


def _empty_like(t, other):
    if other is None:
        return torch.empty_like(t, memory_format=torch.contiguous_format)
    with torch.cuda.stream(other):
        return torch.empty_like(t, memory_format=torch.contiguous_format)


def _scratch(like, nbytes: int, other):
    """nbytes of scratch, at least 16."""
    return _empty(like, (max(16, nbytes + like.element_size()) // like.element_size(),), like.dtype, other)


def _code(t, name: str) -> int:
    code = _CODES.get(t.dtype)
    if code is None:
        raise ValueError(f"{name}: float32 or bfloat16, not {t.dtype}")
    return code


def _row_stride(t, name: str, rows: int, cols: int) -> int:
    """Row stride of a [rows][cols] tensor with contiguous rows."""
    if t.dim() != 2 or t.shape[0] != rows or t.shape[1] != cols:
        raise ValueError(f"{name}: shape {tuple(t.shape)} where ({rows}, {cols}) is wanted")
    stride, inner = t.stride()
    if inner != 1 and cols > 1:
        raise ValueError(f"{name}: the values of a row have to be contiguous")
    return stride if rows > 1 else max(stride, cols)


def _vector(t, name: str, n: int):
    if t is None:
        return None
    if t.dtype != torch.float32 or t.dim() != 1 or t.shape[0] != n or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous float32 tensor [{n}]")
    return t.data_ptr()


def layer_norm_forward(x, weight=None, bias=None, eps: float = 1e-5, out=None, stream=None):
    """Layer normalisation of the rows of x [rows][cols] (float32 or bfloat16; rows may be strided) with
    float32 weight and bias [cols] or None.  Returns (y, mean, rstd)."""
    handle, other = _place(stream, x, weight, bias, out)
    if x.dim() != 2:
        raise ValueError(f"x: [rows][cols], not {tuple(x.shape)}")
    rows, cols = x.shape
    if cols > _INT_MAX:
        raise ValueError(f"x: {cols} columns")
    code = _code(x, "x")
    xs = _row_stride(x, "x", rows, cols)
    w, b = _vector(weight, "weight", cols), _vector(bias, "bias", cols)
    if out is None:
        y, ys = _empty_like(x, other), cols
    else:
        y, ys = out, _row_stride(out, "out", rows, cols)
        if out.dtype != x.dtype:
            raise ValueError("out: the type of x")
    mean = _empty(x, (rows,), torch.float32, other)
    rstd = _empty_like(mean, other)
    rc = lib().cdgrab_layer_norm_forward(rows, cols, code, x.data_ptr(), xs, w, b, eps, y.data_ptr(), ys, mean.data_ptr(),
                                         rstd.data_ptr(), handle)
    if rc:
        _check(rc, "cdgrab_layer_norm_forward")
    return y, mean, rstd


def layer_norm_backward(dy, x, weight, mean, rstd, dweight=None, dbias=None, dx=None, stream=None):
    """Backward pass of layer_norm_forward for m workers' rows: dy, x [m * rows][cols]; dweight and dbias
    [m][cols] (float32 or bfloat16, equal row strides, views into the gather buffer as a rule) receive each
    worker's own sums, either may be None.  Returns dx."""
    handle, other = _place(stream, dy, x, weight, mean, rstd, dweight, dbias, dx)
    if x.dim() != 2:
        raise ValueError(f"x: [rows][cols], not {tuple(x.shape)}")
    rows, cols = x.shape
    if cols > _INT_MAX:
        raise ValueError(f"x: {cols} columns")
    code = _code(x, "x")
    if dy.dtype != x.dtype:
        raise ValueError("dy: the type of x")
    g = dweight if dweight is not None else dbias
    m, gcode, ws, pw, pb = 1, F32, cols, None, None
    if g is not None:
        m = g.shape[0]
        if m < 1 or rows % m:
            raise ValueError(f"{rows} rows are not {m} workers' equal shares")
        gcode, ws = _code(g, "dweight, dbias"), _row_stride(g, "dweight, dbias", m, cols)
        if dweight is not None:
            pw = dweight.data_ptr()
        if dbias is not None:
            pb = dbias.data_ptr()
            # (with one worker the row stride is not used)
            if dbias is not g and (dbias.dtype != g.dtype or (_row_stride(dbias, "dbias", m, cols) != ws and m > 1)):
                raise ValueError("dweight and dbias: one type and one row stride")
    if dx is None:
        dx, dxs = _empty_like(x, other), cols
    else:
        dxs = _row_stride(dx, "dx", rows, cols)
        if dx.dtype != x.dtype:
            raise ValueError("dx: the type of x")
    L = lib()
    nbytes = L.cdgrab_layer_norm_workspace_bytes(m, rows // m, cols)
    scratch = _scratch(x, nbytes, other)
    rc = L.cdgrab_layer_norm_backward(
        m, rows // m, cols, code, dy.data_ptr(), _row_stride(dy, "dy", rows, cols), x.data_ptr(),
        _row_stride(x, "x", rows, cols), _vector(weight, "weight", cols), _vector(mean, "mean", rows),
        _vector(rstd, "rstd", rows), dx.data_ptr(), dxs, gcode, pw, pb, ws, scratch.data_ptr(), max(16, nbytes), handle)
    if rc:
        _check(rc, "cdgrab_layer_norm_backward")
    return dx


def _head_strides(t, name: str, shape):
    """(batch, token, head) strides of a [batch][token][head][head_dim] tensor."""
    if t.dtype != torch.bfloat16 or t.shape != shape:
        raise ValueError(f"{name}: a bfloat16 tensor of shape {tuple(shape)}, not {tuple(t.shape)} {t.dtype}")
    a, b, c, inner = t.stride()
    if inner != 1 and shape[3] > 1:
        raise ValueError(f"{name}: the values of a head have to be contiguous")
    if (a | b | c) & 7:         # an axis of length one has no stride of its own
        a, b, c = ((v + 7) & ~7 if n <= 1 else v for v, n in zip((a, b, c), shape))
    return a, b, c


_NONE = (0, 0, 0)


def _attention_sizes(q, k, v, causal, scale):
    if q.dim() != 4 or k.dim() != 4:
        raise ValueError("q, k, v: [batch][token][head][head_dim]")
    b, tq, h, d = q.shape
    kb, tk, hk, kd = k.shape
    if kb != b or kd != d:
        raise ValueError("q, k and v do not go together")
    sizes = (b, tq, tk, h, hk, d, 1 if causal else 0, d ** -0.5 if scale is None else scale)
    return sizes, _head_strides(q, "q", q.shape) + _head_strides(k, "k", k.shape) + _head_strides(v, "v", k.shape)


def _lens(t, name: str, batch: int):
    if t is None:
        return None
    if t.dtype != torch.int32 or t.dim() != 1 or t.shape[0] != batch or not t.is_contiguous():
        raise ValueError(f"{name}: an int32 tensor [{batch}]")
    return t.data_ptr()


def attention_forward(q, k, v, causal: bool = False, scale: float | None = None, q_lens=None, kv_lens=None, out=None,
                      stream=None):
    """Softmax attention of q [b][t_q][h][d] with k, v [b][t_kv][h_kv][d], bfloat16, any strides that are
    multiples of 8 (slices of one projection's output).  scale: d**-0.5 by default.  q_lens, kv_lens: int32
    [b], the tokens in use.  Returns (o, lse): o like q, lse float32 [b][h][t_q]."""
    handle, other = _place(stream, q, k, v, q_lens, kv_lens, out)
    sizes, strides = _attention_sizes(q, k, v, causal, scale)
    b, tq, h = sizes[0], sizes[1], sizes[3]
    o = _empty_like(q, other) if out is None else out
    sh = AttentionShape.from_buffer_copy(_SHAPE.pack(*sizes, *strides, *_head_strides(o, "out", q.shape), *_NONE, *_NONE,
                                                     *_NONE, *_NONE))
    lse = _empty(q, (b, h, tq), torch.float32, other)
    rc = lib().cdgrab_attention_forward(sh, q.data_ptr(), k.data_ptr(), v.data_ptr(), _lens(q_lens, "q_lens", b),
                                        _lens(kv_lens, "kv_lens", b), o.data_ptr(), lse.data_ptr(), handle)
    if rc:
        _check(rc, "cdgrab_attention_forward")
    return o, lse


def attention_backward(do, q, k, v, o, lse, causal: bool = False, scale: float | None = None, q_lens=None,
                       kv_lens=None, dq=None, dk=None, dv=None, stream=None):
    """Backward pass of attention_forward from its outputs o and lse and the gradient do of o.
    Returns (dq, dk, dv); destinations may be given (views of one buffer as a rule)."""
    handle, other = _place(stream, do, q, k, v, o, lse, q_lens, kv_lens, dq, dk, dv)
    sizes, strides = _attention_sizes(q, k, v, causal, scale)
    b, tq, h = sizes[0], sizes[1], sizes[3]
    if lse.dtype != torch.float32 or lse.shape != (b, h, tq) or not lse.is_contiguous():
        raise ValueError("lse: a contiguous float32 tensor [batch][heads][len_q]")
    dq = _empty_like(q, other) if dq is None else dq
    dk = _empty_like(k, other) if dk is None else dk
    dv = _empty_like(v, other) if dv is None else dv
    qs, ks = q.shape, k.shape
    sh = AttentionShape.from_buffer_copy(_SHAPE.pack(
        *sizes, *strides, *_head_strides(o, "o", qs), *_head_strides(do, "do", qs), *_head_strides(dq, "dq", qs),
        *_head_strides(dk, "dk", ks), *_head_strides(dv, "dv", ks)))
    L = lib()
    nbytes = L.cdgrab_attention_workspace_bytes(sh)
    scratch = _scratch(q, nbytes, other)
    rc = L.cdgrab_attention_backward(
        sh, do.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(),
        _lens(q_lens, "q_lens", b), _lens(kv_lens, "kv_lens", b), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
        scratch.data_ptr(), max(16, nbytes), handle)
    if rc:
        _check(rc, "cdgrab_attention_backward")
    return dq, dk, dv


def orthogonalise(g, steps: int = 5, coeffs=(3.4445, -4.7750, 2.0315), eps: float = 1e-7, out=None, stream=None):
    """The orthogonalised update of a gradient g [rows][cols] or [batch][rows][cols] (float32 or bfloat16):
    `steps` Newton-Schulz products on g / (|g| + eps).  Coefficients that do not keep singular values out of [0, 1]
    below 234 until the last step are refused.  Returns a bfloat16 tensor of g's shape."""
    handle, other = _place(stream, g, out)
    if g.dim() not in (2, 3):
        raise ValueError("g: [rows][cols] or [batch][rows][cols]")
    rows, cols = g.shape[-2:]
    batch = g.shape[0] if g.dim() == 3 else 1
    if max(batch, rows, cols, abs(steps)) > _INT_MAX:
        raise ValueError(f"g: {tuple(g.shape)}, {steps} steps: beyond 32 bits")
    o = _empty(g, g.shape, torch.bfloat16, other) if out is None else out
    if o.dtype != torch.bfloat16 or o.shape != g.shape:
        raise ValueError("out: a bfloat16 tensor of g's shape")
    if len(coeffs) != 3:
        raise ValueError("coeffs: three numbers")
    strides = []
    for t, name in ((g, "g"), (o, "out")):
        s = t.stride()
        if s[-1] != 1 and cols > 1:
            raise ValueError(f"{name}: the values of a row have to be contiguous")
        strides += [s[0] if len(s) == 3 else 0, s[-2] if rows > 1 else max(cols, s[-2])]
    code = _code(g, "g")
    L = lib()
    nbytes = L.cdgrab_orthogonalise_workspace_bytes(batch, rows, cols)
    scratch = _scratch(g, nbytes, other)
    rc = L.cdgrab_orthogonalise(batch, rows, cols, code, g.data_ptr(), strides[0], strides[1], steps,
                                (C.c_float * 3)(*coeffs), eps, o.data_ptr(), strides[2], strides[3], scratch.data_ptr(),
                                max(16, nbytes), handle)
    if rc:
        _check(rc, "cdgrab_orthogonalise")
    return o


def operators_status() -> int:
    """cdgrab_operators_status: what the training operators' kernels reported so far (read and cleared)."""
    return int(lib().cdgrab_operators_status())


def operators_wait_limit(cycles: int = 0):
    """How long a device-side wait of the calls that follow may last, in SM clock cycles; 0: the default."""
    _check(lib().cdgrab_operators_wait_limit(cycles), "cdgrab_operators_wait_limit")


class ShardedCdGrab:
    """One rank of a column-sharded order server over ``torch.distributed``: this rank owns
    d_local columns; every step all-reduces m*m + m doubles (NCCL on GPUs)."""

    def __init__(self, m: int, n: int, d_local: int, dtype="f32", group=None):
        self.group = group
        self._attach(CdGrab(m, n, d_local, dtype, shard=True), m, "cuda")

    def _attach(self, handle, m: int, device):
        """The shard handle this rank drives and the buffer its partial (G, b) is exchanged in."""
        import torch
        self.h = handle
        self.gram = torch.empty(m * m + m, dtype=torch.float64, device=device)

    def begin_epoch(self):
        self.h.begin_epoch()

    def step(self, grads_local):
        import torch.distributed as dist
        self.h.step_begin(grads_local, self.gram)
        if dist.is_available() and dist.is_initialized() and dist.get_world_size(self.group) > 1:
            dist.all_reduce(self.gram, op=dist.ReduceOp.SUM, group=self.group)
        self.h.step_finish(grads_local, self.gram)

    def end_epoch(self, perms_out=None):
        self.h.end_epoch(perms_out)

    def destroy(self):
        self.h.destroy()
