"""Thin Python binding of the C ABI in include/loract.h: argument marshalling only.

Every function takes torch tensors that already live on the GPU (torch supplies device memory
and the current HIP stream), checks shapes and dtypes, and forwards raw pointers to the
library.  Names match the C entry points.  No step of the method runs in Python.
"""
from __future__ import annotations

import ctypes
import operator
import struct
from typing import Dict, NamedTuple, Optional, Sequence, Tuple

import torch

from . import _lib
from ._lib import LoractParams

F32, BF16 = 0, 1
MAX_RANK = 320
STATUS_RANK_DEFICIENT = 1
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
W_OUT_IN, W_IN_OUT = 0, 1
MAX_LORA_RANK = 64
MAX_HEAD = 1024


class LoractError(RuntimeError):
    def __init__(self, code: int, where: str):
        lib = _lib.load()
        msg = lib.loract_strerror(code).decode()
        hip = lib.loract_last_hip_error().decode()
        super().__init__("%s failed: %s (%d)%s" % (where, msg, code, (" [" + hip + "]") if hip else ""))
        self.code = code


def _check(code: int, where: str) -> None:
    if code != 0:
        raise LoractError(code, where)


_DTYPE_CODES = {torch.float32: F32, torch.bfloat16: BF16}


def _dtype_code(dt: torch.dtype) -> int:
    code = _DTYPE_CODES.get(dt)
    if code is None:
        raise TypeError("unsupported dtype %s (float32 or bfloat16)" % dt)
    return code


def _torch_dtype(code: int) -> torch.dtype:
    return torch.bfloat16 if code == BF16 else torch.float32


def _stream_ptr() -> int:
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _require_cuda(*tensors: torch.Tensor) -> None:
    for t in tensors:
        if not t.is_cuda:
            raise ValueError("tensors must live on the GPU")


_workspaces: Dict[Tuple[int, int], torch.Tensor] = {}


def _workspace(nbytes: int, device: torch.device) -> torch.Tensor:
    """A uint8 device buffer of at least `nbytes`, to be held until the call that takes it has been enqueued: the stream's cached one
    (grown on demand, never shrunk), or while the stream is being captured one of the graph's own memory.  The cached one
    is replaced when it grows and is the eager calls', and replays use the address that they were captured with."""
    if torch._C._cuda_isCurrentStreamCapturing():
        return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)
    key = (device.index if device.index is not None else torch.cuda.current_device(), _stream_ptr())
    ws = _workspaces.get(key)
    if ws is None or ws.numel() < nbytes:
        ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)
        _workspaces[key] = ws
    return ws


def loract_version() -> str:
    return _lib.load().loract_version().decode()


def loract_sample_indices(m: int, l: int, seed: int) -> list:
    """Algorithm 1, row sampling (host): the l ascending distinct row ids for `seed`."""
    buf = (ctypes.c_int32 * max(l, 1))()
    _check(_lib.load().loract_sample_indices(m, l, seed & (2 ** 64 - 1), buf), "loract_sample_indices")
    return [int(buf[i]) for i in range(l)]


def make_params(x: torch.Tensor, k: int, l: int = 0, t: int = 0, seed: int = 0,
                factor_dtype: Optional[torch.dtype] = None) -> LoractParams:
    if x.dim() != 2 or x.stride(1) != 1:
        raise ValueError("X must be a 2-D tensor with unit column stride")
    fd = x.dtype if factor_dtype is None else factor_dtype
    return LoractParams(m=x.shape[0], n=x.shape[1], ldx=x.stride(0) if x.shape[0] > 1 else x.shape[1],
                        k=k, l=l, t=t, x_dtype=_dtype_code(x.dtype), factor_dtype=_dtype_code(fd),
                        seed=seed & (2 ** 64 - 1))


def loract_workspace_bytes(params: LoractParams) -> int:
    out = ctypes.c_size_t(0)
    _check(_lib.load().loract_workspace_bytes(ctypes.byref(params), ctypes.byref(out)),
           "loract_workspace_bytes")
    return int(out.value)


def loract_compress(x: torch.Tensor, k: int, t: int = 0, seed: int = 0,
                    idx: Optional[Sequence[int]] = None,
                    factor_dtype: Optional[torch.dtype] = None,
                    out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None,
                    status: Optional[torch.Tensor] = None, l: int = 0
                    ) -> Tuple[torch.Tensor, torch.Tensor]:
    """U (m x k), V (k x n) of Algorithm 1 for the GPU matrix `x`; enqueued on the current stream.

    `l` > k samples l rows (Theorem 4.3) and cuts the result to rank k; 0 means l = k.
    """
    _require_cuda(x)
    lib = _lib.load()
    p = make_params(x, k, l, t, seed, factor_dtype)
    fdt = _torch_dtype(p.factor_dtype)
    if out is None:
        u = torch.empty((p.m, k), dtype=fdt, device=x.device)
        v = torch.empty((k, p.n), dtype=fdt, device=x.device)
    else:
        u, v = out
        if u.shape != (p.m, k) or v.shape != (k, p.n) or u.dtype != fdt or v.dtype != fdt \
                or not u.is_contiguous() or not v.is_contiguous():
            raise ValueError("out=(U, V) must be contiguous m x k and k x n tensors of the factor dtype")
    ws = _workspace(loract_workspace_bytes(p), x.device)
    idx_arr = None
    if idx is not None:
        n_idx = l if l else k
        if len(idx) != n_idx:
            raise ValueError("idx must hold l row ids (k when l is 0)")
        idx_arr = (ctypes.c_int32 * n_idx)(*[int(i) for i in idx])
    if status is not None and (status.dtype != torch.int32 or not status.is_cuda):
        raise ValueError("status must be an int32 GPU tensor")
    _check(lib.loract_compress(x.data_ptr(), ctypes.byref(p), idx_arr, u.data_ptr(), v.data_ptr(),
                               ws.data_ptr(), ws.numel(), _stream_ptr(),
                               status.data_ptr() if status is not None else None),
           "loract_compress")
    return u, v


def loract_compress_adaptive(x: torch.Tensor, k_max: int, energy: float = 0.9, l: int = 0, t: int = 0,
                             seed: int = 0, idx: Optional[Sequence[int]] = None,
                             factor_dtype: Optional[torch.dtype] = None,
                             status: Optional[torch.Tensor] = None
                             ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """Algorithm 1 with the rank chosen by the retained-energy count of Section 2 (sum of singular
    values of the l x n factor), at most k_max.  Returns U (m x k_max), V (k_max x n) whose columns /
    rows from the chosen rank on are zero, and the chosen rank as an int32 GPU tensor (read it when
    convenient: nothing here synchronises)."""
    _require_cuda(x)
    lib = _lib.load()
    p = make_params(x, k_max, l, t, seed, factor_dtype)
    fdt = _torch_dtype(p.factor_dtype)
    u = torch.empty((p.m, k_max), dtype=fdt, device=x.device)
    v = torch.empty((k_max, p.n), dtype=fdt, device=x.device)
    k_out = torch.zeros((1,), dtype=torch.int32, device=x.device)
    ws = _workspace(loract_workspace_bytes(p), x.device)
    idx_arr = None
    if idx is not None:
        n_idx = l if l else k_max
        if len(idx) != n_idx:
            raise ValueError("idx must hold l row ids (k_max when l is 0)")
        idx_arr = (ctypes.c_int32 * n_idx)(*[int(i) for i in idx])
    if status is not None and (status.dtype != torch.int32 or not status.is_cuda):
        raise ValueError("status must be an int32 GPU tensor")
    _check(lib.loract_compress_adaptive(x.data_ptr(), ctypes.byref(p), idx_arr, float(energy), u.data_ptr(),
                                        v.data_ptr(), k_out.data_ptr(), ws.data_ptr(), ws.numel(),
                                        _stream_ptr(), status.data_ptr() if status is not None else None),
           "loract_compress_adaptive")
    return u, v, k_out


def loract_reconstruct(u: torch.Tensor, v: torch.Tensor, out_dtype: Optional[torch.dtype] = None,
                       out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Xhat = U V (Section 3.1, Eq. 4)."""
    _require_cuda(u, v)
    if u.dim() != 2 or v.dim() != 2 or u.shape[1] != v.shape[0] or u.dtype != v.dtype:
        raise ValueError("need U (m x k) and V (k x n) of one dtype")
    if not u.is_contiguous() or not v.is_contiguous():
        raise ValueError("U and V must be contiguous")
    m, k = u.shape
    n = v.shape[1]
    odt = u.dtype if out_dtype is None else out_dtype
    if out is None:
        out = torch.empty((m, n), dtype=odt, device=u.device)
    elif out.shape != (m, n) or out.dtype != odt or out.stride(1) != 1:
        raise ValueError("out must be an m x n tensor of the output dtype with unit column stride")
    _check(_lib.load().loract_reconstruct(u.data_ptr(), v.data_ptr(), m, n, k, _dtype_code(u.dtype),
                                          out.data_ptr(), out.stride(0) if m > 1 else n,
                                          _dtype_code(odt), _stream_ptr()),
           "loract_reconstruct")
    return out


def loract_lora_grad(u: torch.Tensor, v: torch.Tensor, dy: torch.Tensor, b_lora: torch.Tensor,
                     scale: float = 1.0, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """dA = (U V)^T (dY B_lora^T) * scale, n x r float32, without forming U V."""
    _require_cuda(u, v, dy, b_lora)
    m, k = u.shape
    n = v.shape[1]
    if v.shape[0] != k or dy.shape[0] != m or b_lora.shape[1] != dy.shape[1] or u.dtype != v.dtype \
            or dy.dtype != b_lora.dtype:
        raise ValueError("shape or dtype mismatch")
    for tns in (u, v, dy, b_lora):
        if not tns.is_contiguous():
            raise ValueError("operands must be contiguous")
    n_out, r = dy.shape[1], b_lora.shape[0]
    lib = _lib.load()
    nbytes = ctypes.c_size_t(0)
    _check(lib.loract_lora_grad_workspace_bytes(m, n, k, n_out, r, ctypes.byref(nbytes)),
           "loract_lora_grad_workspace_bytes")
    ws = _workspace(int(nbytes.value), u.device)
    if out is None:
        out = torch.empty((n, r), dtype=torch.float32, device=u.device)
    elif out.shape != (n, r) or out.dtype != torch.float32 or not out.is_contiguous():
        raise ValueError("out must be a contiguous n x r float32 tensor")
    _check(lib.loract_lora_grad(u.data_ptr(), v.data_ptr(), m, n, k, _dtype_code(u.dtype),
                                dy.data_ptr(), n_out, b_lora.data_ptr(), r, _dtype_code(dy.dtype),
                                float(scale), out.data_ptr(), ws.data_ptr(), ws.numel(), _stream_ptr()),
           "loract_lora_grad")
    return out


def loract_lora_grad_static(u: torch.Tensor, v: torch.Tensor, dy: torch.Tensor, b_lora: torch.Tensor,
                            out: torch.Tensor, scale: float = 1.0) -> torch.Tensor:
    """loract_lora_grad on the scratch buffer built into the library: nothing is allocated, here or
    in the library, so `out` (n x r float32) must be given.  Shapes that need more than
    loract_static_scratch_bytes() of scratch raise LoractError."""
    _require_cuda(u, v, dy, b_lora, out)
    m, k = u.shape
    n = v.shape[1]
    if v.shape[0] != k or dy.shape[0] != m or b_lora.shape[1] != dy.shape[1] or u.dtype != v.dtype \
            or dy.dtype != b_lora.dtype:
        raise ValueError("shape or dtype mismatch")
    for tns in (u, v, dy, b_lora, out):
        if not tns.is_contiguous():
            raise ValueError("operands must be contiguous")
    n_out, r = dy.shape[1], b_lora.shape[0]
    if out.shape != (n, r) or out.dtype != torch.float32:
        raise ValueError("out must be a contiguous n x r float32 tensor")
    _check(_lib.load().loract_lora_grad_static(
        u.data_ptr(), v.data_ptr(), m, n, k, _dtype_code(u.dtype), dy.data_ptr(), n_out,
        b_lora.data_ptr(), r, _dtype_code(dy.dtype), float(scale), out.data_ptr(), _stream_ptr()),
        "loract_lora_grad_static")
    return out


def loract_static_scratch_bytes() -> int:
    return int(_lib.load().loract_static_scratch_bytes())


def loract_gaussian_omega_t(l: int, n: int, dtype: torch.dtype, seed: int,
                            device: Optional[torch.device] = None) -> torch.Tensor:
    """The comparator's Gaussian test matrix, stored transposed (l x n), generated on the GPU."""
    device = torch.device("cuda", torch.cuda.current_device()) if device is None else device
    out = torch.empty((l, n), dtype=dtype, device=device)
    _check(_lib.load().loract_gaussian_omega_t(out.data_ptr(), l, n, _dtype_code(dtype),
                                               seed & (2 ** 64 - 1), _stream_ptr()),
           "loract_gaussian_omega_t")
    return out


def loract_rsvd(x: torch.Tensor, k: int, oversample: int = 0, power_iters: int = 0, seed: int = 0,
                omega_t: Optional[torch.Tensor] = None,
                factor_dtype: Optional[torch.dtype] = None,
                status: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Randomized-SVD comparator (Section 3.2): rank-k factors U (m x k), V (k x n)."""
    _require_cuda(x)
    lib = _lib.load()
    l = k + oversample
    p = make_params(x, k, l, power_iters, seed, factor_dtype)
    fdt = _torch_dtype(p.factor_dtype)
    if omega_t is not None:
        _require_cuda(omega_t)
        if omega_t.shape != (l, p.n) or omega_t.dtype != x.dtype or not omega_t.is_contiguous():
            raise ValueError("omega_t must be a contiguous l x n tensor of X's dtype")
    u = torch.empty((p.m, k), dtype=fdt, device=x.device)
    v = torch.empty((k, p.n), dtype=fdt, device=x.device)
    ws = _workspace(loract_workspace_bytes(p), x.device)
    _check(lib.loract_rsvd(x.data_ptr(), ctypes.byref(p),
                           omega_t.data_ptr() if omega_t is not None else None,
                           u.data_ptr(), v.data_ptr(), ws.data_ptr(), ws.numel(), _stream_ptr(),
                           status.data_ptr() if status is not None else None),
           "loract_rsvd")
    return u, v


def loract_prenorm_forward(x: torch.Tensor, gamma: torch.Tensor, eps: float = 0.0
                           ) -> Tuple[torch.Tensor, torch.Tensor]:
    """Section 3.3, Eqs. (6)-(7): A = X / RMS(X) * gamma and the RMS vector (float32, m)."""
    _require_cuda(x, gamma)
    if x.dim() != 2 or x.stride(1) != 1 or gamma.dtype != torch.float32 or gamma.numel() != x.shape[1] \
            or not gamma.is_contiguous():
        raise ValueError("need a 2-D X with unit column stride and a contiguous float32 gamma of length n")
    m, n = x.shape
    a = torch.empty((m, n), dtype=x.dtype, device=x.device)
    rms = torch.empty((m,), dtype=torch.float32, device=x.device)
    _check(_lib.load().loract_prenorm_forward(x.data_ptr(), m, n, x.stride(0) if m > 1 else n,
                                              _dtype_code(x.dtype), gamma.data_ptr(), float(eps),
                                              a.data_ptr(), n, rms.data_ptr(), _stream_ptr()),
           "loract_prenorm_forward")
    return a, rms


def loract_prenorm_backward(a: torch.Tensor, rms: torch.Tensor, gamma: torch.Tensor,
                            grad_a: torch.Tensor) -> torch.Tensor:
    """Section 3.3, Eqs. (8)-(10): dL/dX from the (reconstructed) A, the RMS vector and dL/dA."""
    _require_cuda(a, rms, gamma, grad_a)
    if a.shape != grad_a.shape or a.dtype != grad_a.dtype or a.stride(1) != 1 or grad_a.stride(1) != 1:
        raise ValueError("A and dA must have the same shape and dtype, unit column stride")
    m, n = a.shape
    if rms.dtype != torch.float32 or rms.numel() != m or gamma.dtype != torch.float32 or gamma.numel() != n:
        raise ValueError("rms (m) and gamma (n) must be float32")
    dx = torch.empty((m, n), dtype=a.dtype, device=a.device)
    _check(_lib.load().loract_prenorm_backward(a.data_ptr(), m, n, a.stride(0) if m > 1 else n,
                                               _dtype_code(a.dtype), rms.data_ptr(), gamma.data_ptr(),
                                               grad_a.data_ptr(), grad_a.stride(0) if m > 1 else n,
                                               dx.data_ptr(), n, _stream_ptr()),
           "loract_prenorm_backward")
    return dx


# The parameter structures of the sub-layer's entry points as bytes (loract_linear_params, loract_qk_params): a call in
# serving is a few microseconds, and packing is a tenth of filling a ctypes structure.
_LINEAR_PARAMS = struct.Struct("9q5ifdQ")
_QK_PARAMS = struct.Struct("q6iqf4x12q")
_SEED = 2 ** 64 - 1
_DTYPE_OF = operator.attrgetter("dtype")
_WORKSPACE_TOO_SMALL = -2


def _stream_on(device: int) -> int:
    """The current stream of the GPU that a call's tensors live on, which must be the current one: there the kernels run."""
    if torch._C._cuda_getDevice() != device:
        raise ValueError("the tensors live on GPU %d, which is not the current one" % device)
    return torch._C._cuda_getCurrentRawStream(device)


def _rows(t: torch.Tensor, rows: int, cols: int, dtype: torch.dtype, what: str, device: int) -> int:
    """Leading dimension of a matrix of that shape and type with unit column stride on that GPU (negative: none)."""
    if t.shape != (rows, cols) or t.dtype is not dtype or t.get_device() != device or device < 0:
        raise ValueError("%s must be a %d x %d tensor of %s on one GPU with the others" % (what, rows, cols, dtype))
    ld, step = t.stride()
    if step != 1 and cols > 1:
        raise ValueError("%s must have unit column stride" % what)
    if rows < 2:
        return cols
    if ld < cols:
        raise ValueError("the rows of %s must not overlap" % what)
    return ld


def _floats(t: Optional[torch.Tensor], n: int, what: str, device: int) -> Optional[int]:
    if t is None:
        return None
    if t.shape != (n,) or t.dtype is not torch.float32 or not t.is_contiguous() or t.get_device() != device:
        raise ValueError("%s must be a contiguous float32 tensor of length %d on one GPU with the others" % (what, n))
    return t.data_ptr()


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _enqueue(call, args: tuple, query, params: bytes, device: int, where: str) -> None:
    """call(*args, workspace, its bytes, stream) on the stream's cached workspace, or where that is too small (which a call says before it
    enqueues anything) or the stream is being captured on one of the size that `query` gives (None: the call needs none)."""
    stream = _stream_on(device)
    held = None if query is None or torch._C._cuda_isCurrentStreamCapturing() else _workspaces.get((device, stream))
    code = call(*args, None, 0, stream) if held is None else call(*args, held.data_ptr(), held.numel(), stream)
    if code == _WORKSPACE_TOO_SMALL:
        nbytes = ctypes.c_size_t()
        _check(query(params, ctypes.byref(nbytes)), where + "_workspace_bytes")
        held = _workspace(nbytes.value, torch.device("cuda", device))
        code = call(*args, held.data_ptr(), held.numel(), stream)
    if code:
        raise LoractError(code, where)


def _act_code(act: str) -> int:
    code = ACTIVATIONS.get(act)
    if code is None:
        raise ValueError("act must be one of %s" % ", ".join(ACTIVATIONS))
    return code


def loract_dropout(x: torch.Tensor, p_drop: float, seed: int, residual: Optional[torch.Tensor] = None,
                   out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """D(x) + residual, the mask a function of (seed, row, column) that is never stored; the gradient of D is the same
    call on the gradient.  `out` may be x or residual."""
    if x.dim() != 2:
        raise ValueError("x must be a matrix")
    m, n = x.shape
    dt, dev = x.dtype, x.get_device()
    ldx = _rows(x, m, n, dt, "x", dev)
    ldr = 0 if residual is None else _rows(residual, m, n, dt, "residual", dev)
    if out is None:
        out, ldy = x.new_empty((m, n)), n
    else:
        ldy = _rows(out, m, n, dt, "out", dev)
    if m == 0 or n == 0:
        return out
    code = _lib.load().loract_dropout(x.data_ptr(), ldx, _ptr(residual), ldr, m, n, _dtype_code(dt), p_drop, seed & _SEED,
                                      out.data_ptr(), ldy, _stream_on(dev))
    if code:
        raise LoractError(code, "loract_dropout")
    return out


def loract_linear(x: torch.Tensor, w: torch.Tensor, bias: Optional[torch.Tensor] = None, *, w_transposed: bool = False,
                  lora_t: Optional[torch.Tensor] = None, lora_b: Optional[torch.Tensor] = None, lora_scale: float = 1.0,
                  act: str = "none", p_drop: float = 0.0, seed: int = 0, residual: Optional[torch.Tensor] = None,
                  save_preact: bool = False, out_dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None):
    """Y = residual + D(act(P)), P = x w^T + lora_scale lora_t lora_b + bias.

    x m x n_in; w n_out x n_in, or n_in x n_out with `w_transposed` (the forward's weights, for the input gradient);
    bias n_out floats; lora_t m x r and lora_b r x n_out; act none, relu, gelu or silu.  Returns Y, or (Y, Z) with
    `save_preact`: Z = P rounded to x's type, for loract_linear_backward.  `out` may be residual, but share no memory with the others."""
    if x.dim() != 2 or w.dim() != 2:
        raise ValueError("x and w must be matrices")
    m, n_in = x.shape
    n_out = w.shape[1 if w_transposed else 0]
    dt, dev = x.dtype, x.get_device()
    odt = dt if out_dtype is None else out_dtype
    ldx = _rows(x, m, n_in, dt, "x", dev)
    ldw = _rows(w, n_in, n_out, dt, "w", dev) if w_transposed else _rows(w, n_out, n_in, dt, "w", dev)
    r, t_ptr, b_ptr = 0, None, None
    if lora_t is not None or lora_b is not None:
        if lora_t is None or lora_b is None:
            raise ValueError("lora_t and lora_b go together")
        r = lora_b.shape[0]
        if _rows(lora_t, m, r, dt, "lora_t", dev) != r or _rows(lora_b, r, n_out, dt, "lora_b", dev) != n_out:
            raise ValueError("lora_t and lora_b must be contiguous")
        t_ptr, b_ptr = lora_t.data_ptr(), lora_b.data_ptr()
    ldr, r_ptr = (0, None) if residual is None else (_rows(residual, m, n_out, dt, "residual", dev), residual.data_ptr())
    bias_ptr = None if bias is None else _floats(bias, n_out, "bias", dev)
    if out is None:
        out, ldy = x.new_empty((m, n_out)) if odt is dt else x.new_empty((m, n_out), dtype=odt), n_out
    else:
        ldy = _rows(out, m, n_out, odt, "out", dev)
    z = x.new_empty((m, n_out)) if save_preact else None
    if m:
        params = _LINEAR_PARAMS.pack(m, n_in, n_out, ldx, ldw, ldr, ldy, n_out, 0, _dtype_code(dt), _dtype_code(odt),
                                     W_IN_OUT if w_transposed else W_OUT_IN, _act_code(act), r, lora_scale, p_drop, seed & _SEED)
        lib = _lib.load()
        _enqueue(lib.loract_linear, (x.data_ptr(), w.data_ptr(), bias_ptr, t_ptr, b_ptr, r_ptr, params, out.data_ptr(), _ptr(z)),
                 lib.loract_linear_workspace_bytes, params, dev, "loract_linear")
    return (out, z) if save_preact else out


def loract_linear_backward(dy: torch.Tensor, z: Optional[torch.Tensor] = None, *, lora_t: Optional[torch.Tensor] = None,
                           lora_scale: float = 1.0, act: str = "none", p_drop: float = 0.0, seed: int = 0,
                           bias_grad: bool = True, out: Optional[torch.Tensor] = None
                           ) -> Tuple[torch.Tensor, Optional[torch.Tensor], Optional[torch.Tensor]]:
    """dP = act'(z) D(dy), the bias gradient (n_out floats; None without `bias_grad`) and lora_scale lora_t^T dP
    (r x n_out floats; None without `lora_t`), in one pass.  z is what loract_linear kept with `save_preact`; it may
    be None without an activation.  `out` (dP) may be dy or z."""
    if dy.dim() != 2:
        raise ValueError("dy must be a matrix")
    m, n = dy.shape
    dt, dev = dy.dtype, dy.get_device()
    ldy = _rows(dy, m, n, dt, "dy", dev)
    act_code, ldz, z_ptr = _act_code(act), 0, None
    if act_code:
        if z is None:
            raise ValueError("the slope of an activation needs z")
        ldz, z_ptr = _rows(z, m, n, dt, "z", dev), z.data_ptr()
    if out is None:
        out, ldp = dy.new_empty((m, n)), n
    else:
        ldp = _rows(out, m, n, dt, "out", dev)
    db = dy.new_empty((n,), dtype=torch.float32) if bias_grad else None
    r, t_ptr, d_b = 0, None, None
    if lora_t is not None:
        r = lora_t.shape[1] if lora_t.dim() == 2 else 0
        if _rows(lora_t, m, r, dt, "lora_t", dev) != r:
            raise ValueError("lora_t must be contiguous")
        t_ptr, d_b = lora_t.data_ptr(), dy.new_empty((r, n), dtype=torch.float32)
    if m == 0:
        return out, db if db is None else db.zero_(), d_b if d_b is None else d_b.zero_()
    params = _LINEAR_PARAMS.pack(m, 1, n, 0, 0, 0, ldy, ldz, ldp, _dtype_code(dt), 0, 0, act_code, r, lora_scale, p_drop, seed & _SEED)
    lib = _lib.load()
    _enqueue(lib.loract_linear_backward, (dy.data_ptr(), z_ptr, t_ptr, params, out.data_ptr(), _ptr(db), _ptr(d_b)),
             lib.loract_linear_backward_workspace_bytes if bias_grad or r else None, params, dev, "loract_linear_backward")
    return out, db, d_b


def loract_rope_table(n_pos: int, rot: int, theta: float = 10000.0, first: int = 0,
                      device: Optional[torch.device] = None) -> torch.Tensor:
    """Cosines and sines of positions first .. first + n_pos - 1: n_pos x 2 x rot / 2 float32, angles in float64."""
    device = torch.device("cuda", torch.cuda.current_device()) if device is None else device
    table = torch.empty((n_pos, 2, rot // 2), dtype=torch.float32, device=device)
    _check(_lib.load().loract_rope_table(table.data_ptr(), n_pos, rot, float(theta), first, _stream_on(table.get_device())), "loract_rope_table")
    return table


def _heads(t: torch.Tensor, m: int, heads: int, d: int, dtype: torch.dtype, what: str, device: int, written: bool = False) -> Tuple[int, int]:
    """Token and head strides of a tensor tokens x heads x d on that GPU with contiguous heads, which must not overlap if `written`."""
    if t.shape != (m, heads, d) or t.dtype is not dtype or t.get_device() != device or device < 0:
        raise ValueError("%s must be a tensor of %d tokens x %d heads x %d of %s on one GPU with the others" % (what, m, heads, d, dtype))
    token, head, step = t.stride()
    if step != 1 and d > 1:
        raise ValueError("the heads of %s must be contiguous" % what)
    if written and ((token < d and m > 1) or (head < d and heads > 1)):
        raise ValueError("the heads of %s must not overlap" % what)
    return token, head


def _qk_call(q, k, gamma_q, gamma_k, table, positions, eps, interleaved, q_out, k_out, dq, dk):
    """Parameters of a call (dq, dk: the gradients of the forward's outputs, or None)."""
    if q.dim() != 3 or (k is not None and k.dim() != 3):
        raise ValueError("q and k must be tokens x heads x head size")
    m, hq, d = q.shape
    dt, dev = q.dtype, q.get_device()
    hk = 0 if k is None else k.shape[1]
    n_pos, rot = 0, 0
    if table is not None:
        if table.dim() != 3 or table.shape[1] != 2 or table.dtype is not torch.float32 or not table.is_contiguous() or table.get_device() != dev:
            raise ValueError("table must come from loract_rope_table (positions x 2 x rot / 2, float32) and live with q")
        n_pos, rot = table.shape[0], 2 * table.shape[2]
    if positions is not None and (positions.shape != (m,) or positions.dtype is not torch.int32 or
                                  not positions.is_contiguous() or positions.get_device() != dev):
        raise ValueError("positions must be a contiguous int32 tensor with one entry per token and live with q")
    strides = _heads(q, m, hq, d, dt, "q", dev)
    strides += (0, 0) if k is None else _heads(k, m, hk, d, dt, "k", dev)
    strides += (hq * d, d) if q_out is None else _heads(q_out, m, hq, d, dt, "out", dev, True)
    strides += (hk * d, d) if k_out is None else _heads(k_out, m, hk, d, dt, "out", dev, True)
    strides += (0, 0) if dq is None else _heads(dq, m, hq, d, dt, "dq_out", dev)
    strides += (0, 0) if dk is None else _heads(dk, m, hk, d, dt, "dk_out", dev)
    params = _QK_PARAMS.pack(m, hq, hk, d, rot, 1 if interleaved else 0, _dtype_code(dt), n_pos, eps, *strides)
    return params, _floats(gamma_q, d, "gamma_q", dev), None if k is None else _floats(gamma_k, d, "gamma_k", dev)


def loract_qknorm_rope_forward(q: torch.Tensor, k: Optional[torch.Tensor], gamma_q: Optional[torch.Tensor],
                               gamma_k: Optional[torch.Tensor], table: Optional[torch.Tensor], *,
                               positions: Optional[torch.Tensor] = None, eps: float = 1e-6, interleaved: bool = False,
                               out: Optional[Tuple[torch.Tensor, Optional[torch.Tensor]]] = None
                               ) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """Rot(x / rms(x) * gamma) of every head of q and k (tokens x heads x d, any token and head stride: slices of a packed
    projection will do).  table from loract_rope_table (None: no rotation); positions int32, negative for padding, None for
    the token's index.  out = (q, k) works in place."""
    qo, ko = (None, None) if out is None else (out[0], None if k is None else out[1])
    if out is not None and (qo is None or (k is not None and ko is None)):
        raise ValueError("out must hold a tensor for q and one for k")
    params, gq, gk = _qk_call(q, k, gamma_q, gamma_k, table, positions, eps, interleaved, qo, ko, None, None)
    if out is None:
        qo, ko = q.new_empty(q.shape), None if k is None else q.new_empty(k.shape)
    if q.shape[0]:
        code = _lib.load().loract_qknorm_rope_forward(q.data_ptr(), _ptr(k), params, gq, gk, _ptr(table), _ptr(positions),
                                                      qo.data_ptr(), _ptr(ko), _stream_on(q.get_device()))
        if code:
            raise LoractError(code, "loract_qknorm_rope_forward")
    return qo, ko


def loract_qknorm_rope_backward(q: torch.Tensor, k: Optional[torch.Tensor], gamma_q: Optional[torch.Tensor],
                                gamma_k: Optional[torch.Tensor], table: Optional[torch.Tensor], dq_out: torch.Tensor,
                                dk_out: Optional[torch.Tensor], *, positions: Optional[torch.Tensor] = None, eps: float = 1e-6,
                                interleaved: bool = False, out: Optional[Tuple[torch.Tensor, Optional[torch.Tensor]]] = None):
    """(dq, dk, dgamma_q, dgamma_k) from the forward's inputs and the gradients of its outputs; the gammas' gradients are
    float32, None where the gamma is.  out = (dq, dk) may be (dq_out, dk_out) or slices of a packed gradient."""
    dq, dk = (None, None) if out is None else (out[0], None if k is None else out[1])
    if dq_out is None or (k is not None and dk_out is None) or (out is not None and (dq is None or (k is not None and dk is None))):
        raise ValueError("gradients must have the shapes of q and k")
    dk_out = None if k is None else dk_out
    params, gq, gk = _qk_call(q, k, gamma_q, gamma_k, table, positions, eps, interleaved, dq, dk, dq_out, dk_out)
    if out is None:
        dq, dk = q.new_empty(q.shape), None if k is None else q.new_empty(k.shape)
    d = q.shape[2]
    dgq = None if gq is None else q.new_empty((d,), dtype=torch.float32)
    dgk = None if gk is None else q.new_empty((d,), dtype=torch.float32)
    if q.shape[0] == 0:
        return dq, dk, dgq if dgq is None else dgq.zero_(), dgk if dgk is None else dgk.zero_()
    dgk_ptr = _ptr(dgk)
    if dgk is not None and k.shape[1] == 0:            # (the library knows no gradient of keys that are not there)
        dgk_ptr = None
        dgk.zero_()
    lib = _lib.load()
    _enqueue(lib.loract_qknorm_rope_backward, (q.data_ptr(), _ptr(k), params, gq, gk, _ptr(table), _ptr(positions), dq_out.data_ptr(),
                                               _ptr(dk_out), dq.data_ptr(), _ptr(dk), _ptr(dgq), dgk_ptr),
             lib.loract_qknorm_rope_workspace_bytes if dgq is not None or dgk_ptr else None, params, q.get_device(), "loract_qknorm_rope_backward")
    return dq, dk, dgq, dgk


ADAMW_BLOCK = 256
_ADAMW_PARAMS = struct.Struct("5dqQ3i4x")


class AdamwState:
    """The moments of a list of tensors, for loract_adamw: one flat tensor each, every tensor's part padded to a multiple of ADAMW_BLOCK.

    bits = 32: `m` and `v` are float32 and `exps` is None.  bits = 8: `m` and `v` are float8_e4m3fn and stand for m and sqrt(v) in units of
    2^(exps - 127), `exps` (blocks x 2, uint8) one for each block of ADAMW_BLOCK elements and moment.  All are plain tensors, to be saved and
    copied into as such."""

    def __init__(self, sizes: Sequence[int], bits: int, device: torch.device):
        if bits not in (8, 32):
            raise ValueError("states are held in 32 or 8 bits")
        self.sizes, self.bits = tuple(sizes), bits
        self._sizes, self._size_words = list(sizes), struct.pack("%dq" % len(self.sizes), *self.sizes)
        self._padded = padded = sum(-(-n // ADAMW_BLOCK) * ADAMW_BLOCK for n in self.sizes)
        dtype = torch.float32 if bits == 32 else torch.uint8
        self.m, self.v = (torch.zeros(padded, dtype=dtype, device=device) for _ in range(2))
        self.exps = None
        if bits == 8:
            self.m, self.v = self.m.view(torch.float8_e4m3fn), self.v.view(torch.float8_e4m3fn)
            self.exps = torch.zeros((padded // ADAMW_BLOCK, 2), dtype=torch.uint8, device=device)


def loract_adamw_state(params: Sequence[torch.Tensor], bits: int = 32) -> AdamwState:
    """The state before the first step (zeros) of loract_adamw on these tensors, in their order."""
    params = list(params)
    if not params:
        raise ValueError("no tensors")
    _require_cuda(*params)
    return AdamwState([p.numel() for p in params], bits, params[0].device)


def _tensor_list(ts: Sequence[torch.Tensor], sizes: list, dtype: torch.dtype, device: int, what: str) -> bytes:
    """The addresses of contiguous tensors of those sizes and that type on that GPU, as an array."""
    T = torch.Tensor
    if len(ts) != len(sizes) or list(map(T.numel, ts)) != sizes:
        raise ValueError("%s must be the state's %d tensors, with its sizes" % (what, len(sizes)))
    n = len(ts)
    if list(map(_DTYPE_OF, ts)).count(dtype) != n or list(map(T.get_device, ts)).count(device) != n or device < 0 or not all(map(T.is_contiguous, ts)):
        raise ValueError("%s must be contiguous tensors of %s on one GPU with the others" % (what, dtype))
    return struct.pack("%dQ" % n, *map(T.data_ptr, ts))


def _scalar(v, dtype: torch.dtype, device: int, what: str):
    """(number, address): one of a number and a tensor of one element."""
    if not isinstance(v, torch.Tensor):
        return v, None
    if v.numel() != 1 or v.dtype is not dtype or v.get_device() != device:
        raise ValueError("%s must be a number or one %s on one GPU with the others" % (what, dtype))
    return 0, v.data_ptr()


def loract_adamw(params: Sequence[torch.Tensor], grads: Sequence[torch.Tensor], state: AdamwState, *, step, lr, betas: Tuple[float, float] = (0.9, 0.999),
                 eps: float = 1e-8, weight_decay: float = 0.01, seed: int = 0, grad_scale: Optional[torch.Tensor] = None,
                 copies: Optional[Sequence[torch.Tensor]] = None) -> None:
    """One step of AdamW on all of `params` (float32 or bfloat16, in place) and `state`.

    `grads` are float32 or bfloat16.  `copies` of float32 parameters get them rounded to bfloat16.  eps is 0 or 2^-126 at least.  step (from 1 on) and lr are numbers, or
    tensors of one element (int64, float32) that are read when the step runs, as `grad_scale` (float32, multiplies the gradients) always is:
    a captured step takes what changes from replay to replay from these.  Each tensor is looked over by every call (half a microsecond);
    parameters that lie in one buffer can be given as one tensor.  What is held in fewer than 32 bits is rounded at random by
    (seed, step), so that small changes are kept on average.

    Like everything that this package writes, parameters and copies change without autograd's notice: a backward pass through a graph that
    saved them before the step does not raise (torch.autograd.graph.increment_version(params) makes it)."""
    params, grads = list(params), list(grads)
    if not params or not grads:
        raise ValueError("no tensors")
    sizes, dev, dt, gdt = state._sizes, params[0].get_device(), params[0].dtype, grads[0].dtype
    p_ptr = _tensor_list(params, sizes, dt, dev, "params")
    g_ptr = _tensor_list(grads, sizes, gdt, dev, "grads")
    c_ptr = None
    if copies is not None:
        if dt is not torch.float32:
            raise ValueError("only float32 parameters have copies")
        c_ptr = _tensor_list(list(copies), sizes, torch.bfloat16, dev, "copies")
    padded = state._padded
    held = torch.float32 if state.bits == 32 else torch.float8_e4m3fn
    for t in (state.m, state.v):
        if t.shape != (padded,) or t.dtype is not held or not t.is_contiguous() or t.get_device() != dev:
            raise ValueError("the state's moments must be contiguous tensors of %d %s on one GPU with the parameters" % (padded, held))
    if state.bits == 8 and (state.exps.shape != (padded // ADAMW_BLOCK, 2) or state.exps.dtype is not torch.uint8 or not state.exps.is_contiguous() or
                            state.exps.get_device() != dev):
        raise ValueError("the state's exponents must be a contiguous blocks x 2 uint8 tensor on one GPU with the parameters")
    lr, lr_ptr = _scalar(lr, torch.float32, dev, "lr")
    step, step_ptr = _scalar(step, torch.int64, dev, "step")
    scale_ptr = None
    if grad_scale is not None:
        if not isinstance(grad_scale, torch.Tensor):
            raise ValueError("grad_scale must be a tensor")
        scale_ptr = _scalar(grad_scale, torch.float32, dev, "grad_scale")[1]
    args = _ADAMW_PARAMS.pack(lr, betas[0], betas[1], eps, weight_decay, step, seed & _SEED, _dtype_code(dt), _dtype_code(gdt), state.bits)
    code = _lib.load().loract_adamw(p_ptr, g_ptr, c_ptr, state._size_words, len(sizes), args, state.m.data_ptr(),
                                    state.v.data_ptr(), _ptr(state.exps), lr_ptr, step_ptr, scale_ptr, _stream_on(dev))
    if code:
        raise LoractError(code, "loract_adamw")


MAX_TOP = 64
_LOGPROB_PARAMS = struct.Struct("4q4id")
_TARGET_BITS = {torch.int32: 32, torch.int64: 64}


class TokenLogprobs(NamedTuple):
    """What loract_token_logprobs gives: `logp` of the targets (None without them), `entropy`, `stats` (3 x m: maximum, log2 of the sum, entropy)
    for the backward pass, and `top_logp`, `top_ids` (m x top, None without any)."""
    logp: Optional[torch.Tensor]
    entropy: torch.Tensor
    stats: torch.Tensor
    top_logp: Optional[torch.Tensor]
    top_ids: Optional[torch.Tensor]


def _logprob_call(logits, targets, temperature, top, ldg):
    """(parameters, the targets' address) of a call."""
    if logits.dim() != 2:
        raise ValueError("logits must be a matrix")
    m, n = logits.shape
    dev = logits.get_device()
    ld = _rows(logits, m, n, logits.dtype, "logits", dev)
    bits, t_ptr = 32, None
    if targets is not None:
        bits = _TARGET_BITS.get(targets.dtype)
        if bits is None or targets.shape != (m,) or not targets.is_contiguous() or targets.get_device() != dev:
            raise ValueError("targets must be a contiguous int32 or int64 tensor with one entry per token and live with the logits")
        t_ptr = targets.data_ptr()
    if n < 1:
        raise ValueError("an empty vocabulary")
    return _LOGPROB_PARAMS.pack(m, n, ld, ldg, _dtype_code(logits.dtype), bits, top, 0, temperature), t_ptr


def loract_token_logprobs(logits: torch.Tensor, targets: Optional[torch.Tensor] = None, *, temperature: float = 1.0, top: int = 0) -> TokenLogprobs:
    """Log probabilities of `targets` (int32 or int64, negative for none) under softmax(logits / temperature), the rows' entropy, and the `top` (at
    most MAX_TOP) largest logits' log probabilities and indices, ties in the order of their indices.  All float32."""
    params, t_ptr = _logprob_call(logits, targets, temperature, top, 0)
    m, dev = logits.shape[0], logits.get_device()
    logp = None if targets is None else logits.new_empty((m,), dtype=torch.float32)
    stats = logits.new_empty((3, m), dtype=torch.float32)
    top_logp, top_ids = (logits.new_empty((m, top), dtype=torch.float32), logits.new_empty((m, top), dtype=torch.int32)) if top > 0 else (None, None)
    if m:
        lib = _lib.load()
        _enqueue(lib.loract_token_logprobs, (logits.data_ptr(), t_ptr, params, _ptr(logp), stats.data_ptr(), _ptr(top_logp), _ptr(top_ids)),
                 lib.loract_token_logprobs_workspace_bytes, params, dev, "loract_token_logprobs")
    return TokenLogprobs(logp, stats[2], stats, top_logp, top_ids)


def _logprob_grads(logits, targets, d_logp, d_entropy, out):
    if d_logp is None and d_entropy is None:
        raise ValueError("a gradient of the log probabilities or of the entropy is needed")
    if d_logp is not None and targets is None:
        raise ValueError("d_logp needs targets")
    if logits.dim() != 2:
        raise ValueError("logits must be a matrix")
    m, n = logits.shape
    dev = logits.get_device()
    pointers = _floats(d_logp, m, "d_logp", dev), _floats(d_entropy, m, "d_entropy", dev)
    if out is None:
        return logits.new_empty((m, n)), n, pointers
    return out, _rows(out, m, n, logits.dtype, "out", dev), pointers


def loract_token_logprobs_backward(logits: torch.Tensor, targets: Optional[torch.Tensor], stats: torch.Tensor, d_logp: Optional[torch.Tensor],
                                   d_entropy: Optional[torch.Tensor] = None, *, temperature: float = 1.0,
                                   out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The logits' gradient from those of logp and entropy (m floats each, or None) and the forward call's `stats`.  `out` may be logits."""
    out, ldg, (lp_ptr, e_ptr) = _logprob_grads(logits, targets, d_logp, d_entropy, out)
    params, t_ptr = _logprob_call(logits, targets, temperature, 0, ldg)
    m, dev = logits.shape[0], logits.get_device()
    if stats.shape != (3, m) or stats.dtype is not torch.float32 or not stats.is_contiguous() or stats.get_device() != dev:
        raise ValueError("stats must come from loract_token_logprobs")
    if m:
        code = _lib.load().loract_token_logprobs_backward(logits.data_ptr(), t_ptr, params, stats.data_ptr(), lp_ptr, e_ptr, out.data_ptr(), _stream_on(dev))
        if code:
            raise LoractError(code, "loract_token_logprobs_backward")
    return out


def loract_token_logprobs_grad(logits: torch.Tensor, targets: Optional[torch.Tensor], d_logp: Optional[torch.Tensor],
                               d_entropy: Optional[torch.Tensor] = None, *, temperature: float = 1.0, out: Optional[torch.Tensor] = None
                               ) -> Tuple[Optional[torch.Tensor], torch.Tensor, torch.Tensor]:
    """(logp, entropy, the logits' gradient) in one call, where the outputs' gradients are known before them: with d_logp = -1 / tokens it is the
    cross-entropy loss, whose value is the mean of -logp.  `out` may be logits."""
    out, ldg, (lp_ptr, e_ptr) = _logprob_grads(logits, targets, d_logp, d_entropy, out)
    params, t_ptr = _logprob_call(logits, targets, temperature, 0, ldg)
    m, dev = logits.shape[0], logits.get_device()
    logp = None if targets is None else logits.new_empty((m,), dtype=torch.float32)
    stats = logits.new_empty((3, m), dtype=torch.float32)
    if m:
        lib = _lib.load()
        _enqueue(lib.loract_token_logprobs_grad, (logits.data_ptr(), t_ptr, params, lp_ptr, e_ptr, _ptr(logp), stats.data_ptr(), out.data_ptr()),
                 lib.loract_token_logprobs_workspace_bytes, params, dev, "loract_token_logprobs_grad")
    return logp, stats[2], out


_REQUESTS_PARAMS = struct.Struct("7q4i")


def loract_lora_requests(x: torch.Tensor, a: torch.Tensor, b: torch.Tensor, ids: torch.Tensor, scales: Optional[torch.Tensor] = None, *,
                         residual: Optional[torch.Tensor] = None, out_dtype: Optional[torch.dtype] = None,
                         out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Y_i = residual_i + scales[ids_i] (x_i a[ids_i]) b[ids_i]: the adapters of many requests beside a shared projection, whose result is the residual.

    x m x n_in; a adapters x n_in x r and b adapters x r x n_out, contiguous (adapters of smaller rank padded with zeros); ids m int32 in any order, negative
    for none; scales float32.  residual and Y are of out_dtype (x's by default); `out` may be residual, whose rows without an adapter then stay."""
    if x.dim() != 2 or a.dim() != 3 or b.dim() != 3:
        raise ValueError("x must be a matrix, a and b adapters x n_in x r and adapters x r x n_out")
    m, n_in = x.shape
    count, _, r = a.shape
    n_out = b.shape[2]
    dt, dev = x.dtype, x.get_device()
    odt = dt if out_dtype is None else out_dtype
    ldx = _rows(x, m, n_in, dt, "x", dev)
    for t, shape, what in ((a, (count, n_in, r), "a"), (b, (count, r, n_out), "b")):
        if t.shape != shape or t.dtype is not dt or not t.is_contiguous() or t.get_device() != dev:
            raise ValueError("%s must be a contiguous %d x %d x %d tensor of %s on one GPU with the others" % ((what,) + shape + (dt,)))
    if ids.shape != (m,) or ids.dtype is not torch.int32 or not ids.is_contiguous() or ids.get_device() != dev:
        raise ValueError("ids must be a contiguous int32 tensor with one entry per token on one GPU with the others")
    s_ptr = _floats(scales, count, "scales", dev)
    ldr, r_ptr = (0, None) if residual is None else (_rows(residual, m, n_out, odt, "residual", dev), residual.data_ptr())
    if out is None:
        out, ldy = x.new_empty((m, n_out), dtype=odt), n_out
    else:
        ldy = _rows(out, m, n_out, odt, "out", dev)
    if m:
        params = _REQUESTS_PARAMS.pack(m, n_in, n_out, count, ldx, ldr, ldy, _dtype_code(dt), _dtype_code(odt), r, 0)
        lib = _lib.load()
        _enqueue(lib.loract_lora_requests, (x.data_ptr(), a.data_ptr(), b.data_ptr(), ids.data_ptr(), s_ptr, r_ptr, params, out.data_ptr()),
                 lib.loract_lora_requests_workspace_bytes, params, dev, "loract_lora_requests")
    return out


def loract_profile_begin() -> None:
    _check(_lib.load().loract_profile_begin(), "loract_profile_begin")


def loract_profile_end() -> Dict[str, Tuple[float, int]]:
    """Stops per-kernel timing; returns {kernel name: (total milliseconds, launches)}."""
    lib = _lib.load()
    _check(lib.loract_profile_end(), "loract_profile_end")
    out: Dict[str, Tuple[float, int]] = {}
    buf = ctypes.create_string_buffer(128)
    for i in range(lib.loract_profile_count()):
        ms = ctypes.c_double(0.0)
        cnt = ctypes.c_int64(0)
        _check(lib.loract_profile_get(i, buf, 128, ctypes.byref(ms), ctypes.byref(cnt)),
               "loract_profile_get")
        out[buf.value.decode()] = (float(ms.value), int(cnt.value))
    return out
