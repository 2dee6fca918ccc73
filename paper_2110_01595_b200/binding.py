"""ctypes binding of libsolon.so: same names as the C interface (include/solon.h), marshalling only.

Torch is used for device memory and streams; every step of the path runs in the library's kernels.
The library is loaded on first use and a missing build raises: there is no fallback of any kind.
"""

from __future__ import annotations

import ctypes
import functools
import os
from ctypes import POINTER, byref, c_char_p, c_double, c_float, c_int, c_int64, c_uint8, c_uint64, c_void_p
from typing import NamedTuple

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsolon.so")

OK = 0
ERR_INVALID_ARG = -1
ERR_INFEASIBLE = -2
ERR_CUDA = -3
ERR_UNDECODABLE = -4
ERR_INTERNAL = -5
ERR_NOMEM = -6
F32 = 0
F64 = 1
BF16 = 2
F16 = 3

# name -> (restype, argtypes); every symbol the header declares
SIGNATURES = {
    "solon_check_params": (c_int, [c_int, c_int, c_int, c_int, c_int64]),
    "solon_group_layout": (c_int, [c_int, c_int, POINTER(c_int), c_int, POINTER(c_int)]),
    "solon_node_scalars": (c_int, [c_int, c_int, POINTER(c_double)]),
    "solon_locate_host": (c_int, [c_int, c_int, c_int, c_int, POINTER(c_double), POINTER(c_double), POINTER(c_double),
                                  c_double, POINTER(c_uint8), POINTER(c_int), POINTER(c_int), POINTER(c_int),
                                  POINTER(c_double)]),
    "solon_strerror": (c_char_p, [c_int]),
    "solon_plan_create": (c_int, [c_int, c_int, c_int, c_int, c_int64, c_uint64, POINTER(c_void_p)]),
    "solon_plan_create_ex": (c_int, [c_int, c_int, c_int, c_int, c_int64, c_uint64, c_int, POINTER(c_void_p)]),
    "solon_float64_m_supported": (c_int, [c_int]),
    "solon_plan_dtype": (c_int, [c_void_p]),
    "solon_plan_destroy": (c_int, [c_void_p]),
    "solon_plan_set_stream": (c_int, [c_void_p, c_void_p]),
    "solon_plan_set_num_projections": (c_int, [c_void_p, c_int]),
    "solon_plan_reseed": (c_int, [c_void_p, c_uint64]),
    "solon_plan_set_fresh_projections": (c_int, [c_void_p, c_int]),
    "solon_plan_set_tolerance": (c_int, [c_void_p, c_double]),
    "solon_plan_set_early_locator": (c_int, [c_void_p, c_int]),
    "solon_plan_set_optimistic": (c_int, [c_void_p, c_int]),
    "solon_plan_get_optimistic_outcome": (c_int, [c_void_p, POINTER(c_int)]),
    "solon_plan_set_lsq_rows": (c_int, [c_void_p, c_int]),
    "solon_plan_dc": (c_int64, [c_void_p]),
    "solon_plan_num_groups": (c_int, [c_void_p]),
    "solon_plan_group_of": (c_int, [c_void_p, c_int]),
    "solon_plan_group_start": (c_int, [c_void_p, c_int]),
    "solon_plan_group_size": (c_int, [c_void_p, c_int]),
    "solon_plan_num_projections": (c_int, [c_void_p]),
    "solon_plan_get_node_scalars": (c_int, [c_void_p, POINTER(c_double)]),
    "solon_plan_get_projection_vectors": (c_int, [c_void_p, POINTER(c_float)]),
    "solon_encode": (c_int, [c_void_p, c_void_p, c_void_p]),
    "solon_decode": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p]),
    "solon_encode_f64": (c_int, [c_void_p, c_void_p, c_void_p]),
    "solon_decode_f64": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p]),
    "solon_overwrite_rows_f64": (c_int, [c_void_p, c_void_p, c_int, c_void_p, c_void_p]),
    "solon_step_host_f64": (c_int, [c_void_p, c_void_p, c_int, POINTER(c_int), c_void_p, c_void_p, c_void_p]),
    "solon_decode_status": (c_int, [c_void_p]),
    "solon_plan_status": (c_int, [c_void_p]),
    "solon_decode_project": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p]),
    "solon_decode_finish": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p]),
    "solon_lsq_grads": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p]),
    "solon_overwrite_rows": (c_int, [c_void_p, c_void_p, c_int, c_void_p, c_void_p]),
    "solon_step_host": (c_int, [c_void_p, c_void_p, c_int, POINTER(c_int), c_void_p, c_void_p, c_void_p]),
    "solon_plan_get_projections": (c_int, [c_void_p, POINTER(c_double), POINTER(c_double)]),
    "solon_plan_get_recovery": (c_int, [c_void_p, POINTER(c_int), POINTER(c_int), POINTER(c_int), POINTER(c_double)]),
    "solon_plan_get_early_outcome": (c_int, [c_void_p, POINTER(c_int)]),
    "solon_plan_kernel_launches": (c_int64, [c_void_p]),
    "solon_plan_set_profiling": (c_int, [c_void_p, c_int]),
    "solon_plan_get_timings": (c_int, [c_void_p, POINTER(c_float)]),
    "solon_layernorm_forward": (c_int, [c_void_p, c_int64, c_int, c_void_p, c_void_p, c_int, c_int64, c_int64, c_double, c_void_p, c_int64, c_void_p,
                                        c_void_p, c_void_p]),
    "solon_layernorm_backward_workspace": (c_int64, [c_int64, c_int64, c_int]),
    "solon_layernorm_backward": (c_int, [c_void_p, c_int64, c_void_p, c_int64, c_int, c_void_p, c_int, c_void_p, c_void_p, c_int64, c_int64, c_int,
                                         c_void_p, c_int64, c_void_p, c_void_p, c_int64, c_int, c_void_p, c_int64, c_void_p]),
    "solon_token_logprobs": (c_int, [c_void_p, c_int64, c_int, c_void_p, c_int64, c_int64, c_int, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                     c_void_p, c_void_p]),
    "solon_token_logprobs_backward": (c_int, [c_void_p, c_int64, c_int, c_void_p, c_int64, c_int64, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                              c_void_p, c_int64, c_void_p]),
    "solon_adamw_state_blocks": (c_int64, [c_int, POINTER(c_int64)]),
    "solon_adamw_create": (c_int, [c_int, POINTER(c_int64), POINTER(c_void_p), POINTER(c_void_p), POINTER(c_float), c_int, c_void_p, c_void_p, c_void_p,
                                   c_double, c_double, c_double, c_uint64, POINTER(c_void_p)]),
    "solon_adamw_destroy": (c_int, [c_void_p]),
    "solon_adamw_bind_grads": (c_int, [c_void_p, POINTER(c_void_p), c_int]),
    "solon_adamw_step": (c_int, [c_void_p, c_void_p, c_int, c_double, c_double, c_double, c_void_p, c_void_p, c_void_p]),
    "solon_adamw_set_step": (c_int, [c_void_p, c_int64]),
    "solon_adamw_get_steps": (c_int, [c_void_p, POINTER(c_int64), POINTER(c_int64)]),
    "solon_adamw_moments": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p]),
    "solon_project_noalloc": (c_int, [c_void_p, c_void_p, c_int64, c_int, c_int64, c_int, c_void_p, c_void_p, c_void_p]),
}

_lib = None


class SolonError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {strerror(status)} ({status})")


def lib() -> ctypes.CDLL:
    """The loaded library; raises if it has not been built (python -m paper_2110_01595_b200.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2110_01595_b200.build`")
        handle = ctypes.CDLL(LIB_PATH)
        for name, (restype, argtypes) in SIGNATURES.items():
            fn = getattr(handle, name)
            fn.restype = restype
            fn.argtypes = argtypes
        _lib = handle
    return _lib


def strerror(status: int) -> str:
    return lib().solon_strerror(status).decode()


def _check(status: int, where: str) -> None:
    if status != OK:
        raise SolonError(status, where)


def _dptr(a: np.ndarray, ctype):
    return a.ctypes.data_as(POINTER(ctype))


# ------------------------------------------------------------------ plan-free helpers


def solon_check_params(P: int, s: int, m: int, r: int, d: int) -> int:
    return lib().solon_check_params(P, s, m, r, d)


def solon_group_layout(P: int, r: int) -> list[int]:
    starts = np.zeros(P + 2, dtype=np.int32)
    q = c_int(0)
    _check(lib().solon_group_layout(P, r, _dptr(starts, c_int), len(starts), byref(q)), "solon_group_layout")
    return starts[:q.value + 1].tolist()


def solon_node_scalars(P: int, r: int) -> np.ndarray:
    w = np.zeros(P, dtype=np.float64)
    _check(lib().solon_node_scalars(P, r, _dptr(w, c_double)), "solon_node_scalars")
    return w


def solon_locate_host(rho: np.ndarray, nu: np.ndarray, w_g: np.ndarray, m: int, s: int, tau: float):
    """Host mirror of the device locator for one group.  Returns (status, mask, t, rec_rows, coeff[n_rec, m])."""
    rho = np.ascontiguousarray(np.atleast_2d(rho), dtype=np.float64)
    nu = np.ascontiguousarray(nu, dtype=np.float64)
    w_g = np.ascontiguousarray(w_g, dtype=np.float64)
    K, n = rho.shape
    mask = np.zeros(n, dtype=np.uint8)
    rows = np.zeros(n, dtype=np.int32)
    coeff = np.zeros(n * m, dtype=np.float64)
    t = c_int(0)
    n_rec = c_int(0)
    status = lib().solon_locate_host(n, m, s, K, _dptr(rho, c_double), _dptr(nu, c_double), _dptr(w_g, c_double), tau,
                                     _dptr(mask, c_uint8), byref(t), _dptr(rows, c_int), byref(n_rec),
                                     _dptr(coeff, c_double))
    if status not in (OK, ERR_UNDECODABLE):
        raise SolonError(status, "solon_locate_host")
    return status, mask, t.value, rows[:n_rec.value].copy(), coeff[:n_rec.value * m].reshape(n_rec.value, m).copy()


def solon_project_noalloc(received, f, rho, nu, stream=None) -> int:
    """Projections through the entry point that allocates nothing.

    received: P x d_c float32 CUDA tensor; f: K x f_pitch float32 CUDA tensor (f_pitch >= d_c, multiple of 4);
    rho (K x P) and nu (P): float64 CUDA tensors the caller has already allocated.  Returns the status code.
    """
    import torch

    P, d_c = received.shape
    K, f_pitch = f.shape
    for t, dt in ((received, torch.float32), (f, torch.float32), (rho, torch.float64), (nu, torch.float64)):
        if not (t.is_cuda and t.is_contiguous() and t.dtype == dt):
            raise ValueError("solon_project_noalloc takes contiguous CUDA tensors (float32 in, float64 out)")
    if tuple(rho.shape) != (K, P) or tuple(nu.shape) != (P,):
        raise ValueError("rho must be K x P and nu must have P entries")
    stream = stream if stream is not None else torch.cuda.current_stream()
    return lib().solon_project_noalloc(c_void_p(received.data_ptr()), c_void_p(f.data_ptr()), f_pitch, P, d_c, K,
                                       c_void_p(rho.data_ptr()), c_void_p(nu.data_ptr()), c_void_p(stream.cuda_stream))


# ------------------------------------------------------------------ token-model operators (no plan needed)
#
# All of them enqueue on the current stream of the current device, which the tensors have to be on, and return without
# synchronising.  Outputs may be given (to be reused from step to step) or are allocated.  Nothing is recorded for automatic
# differentiation, whatever the inputs' requires_grad: the gradients are calls of their own.

_torch_dtypes = {}


def _dtype_code(dtype) -> int:
    if not _torch_dtypes:
        import torch

        _torch_dtypes.update({torch.float32: F32, torch.float64: F64, torch.bfloat16: BF16, torch.float16: F16})
    code = _torch_dtypes.get(dtype)
    if code is None:
        raise ValueError(f"unsupported element type {dtype}")
    return code


def _current_stream(device) -> int:
    import torch

    index = device.index
    if index != torch.cuda.current_device():
        raise ValueError(f"tensors are on {device}, the current device is cuda:{torch.cuda.current_device()}")
    return torch._C._cuda_getCurrentRawStream(index)      # torch.cuda.current_stream().cuda_stream, a Stream object less (3 us)


def _matrix(t, name: str, like=None):
    """(pointer, pitch) of a CUDA matrix whose rows are contiguous; `like`: a matrix it has to equal in shape, type and place."""
    if like is not None and (t.shape != like.shape or t.dtype != like.dtype or t.device != like.device):
        raise ValueError(f"{name}: expected {tuple(like.shape)} {like.dtype} on {like.device}, got {tuple(t.shape)} {t.dtype} on {t.device}")
    if t.dim() != 2 or not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA matrix (rows x columns)")
    if t.is_contiguous():
        return t.data_ptr(), t.shape[1]
    rows, cols = t.shape
    pitch, step = t.stride()
    if (step != 1 and cols > 1) or (pitch < cols and rows > 1):
        raise ValueError(f"{name}: the elements of a row must be contiguous and rows must not overlap (strides {tuple(t.stride())})")
    return t.data_ptr(), pitch if rows > 1 else cols


def _empty_matrix(like):
    import torch

    return torch.empty_like(like) if like.is_contiguous() else like.new_empty(like.shape)


def _vector(t, name: str, n: int, dtype, device) -> int:
    if t.dim() != 1 or t.numel() != n or t.dtype != dtype or t.device != device or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous vector of {n} {dtype} on {device}, got {tuple(t.shape)} {t.dtype} on {t.device}")
    return t.data_ptr()


def _params(weight, bias, cols: int, x):
    """(weight pointer, bias pointer, type code) of layer norm parameters in float32 or x's type."""
    given = weight if weight is not None else bias
    if given is None:
        return None, None, F32
    code = _dtype_code(given.dtype)
    return (None if weight is None else _vector(weight, "weight", cols, given.dtype, x.device),
            None if bias is None else _vector(bias, "bias", cols, given.dtype, x.device), code)


def solon_layernorm_forward(x, weight=None, bias=None, eps: float = 1e-5, y=None, mean=None, rstd=None):
    """Layer norm of the rows of x (rows x cols; float32, bfloat16 or float16).  Returns (y, mean, rstd): y in x's type, the
    rows' means and reciprocal standard deviations in float32 for solon_layernorm_backward.  Not recorded by autograd."""
    import torch

    px, x_pitch = _matrix(x, "x")
    rows, cols = x.shape
    device, f32 = x.device, torch.float32
    stream = _current_stream(device)
    if y is None:
        y = _empty_matrix(x)
        py, y_pitch = y.data_ptr(), cols
    else:
        py, y_pitch = _matrix(y, "y", x)
    if mean is None and rstd is None:
        mean, rstd = x.new_empty(rows, dtype=f32), x.new_empty(rows, dtype=f32)
        pm, pr = mean.data_ptr(), rstd.data_ptr()
    else:
        mean = x.new_empty(rows, dtype=f32) if mean is None else mean
        rstd = x.new_empty(rows, dtype=f32) if rstd is None else rstd
        pm, pr = _vector(mean, "mean", rows, f32, device), _vector(rstd, "rstd", rows, f32, device)
    pw, pb, code = _params(weight, bias, cols, x)
    _check(lib().solon_layernorm_forward(px, x_pitch, _dtype_code(x.dtype), pw, pb, code, rows, cols, eps, py, y_pitch, pm, pr, stream),
           "solon_layernorm_forward")
    return y, mean, rstd


@functools.lru_cache(maxsize=256)
def _layernorm_workspace(rows: int, cols: int, partitions: int) -> int:
    return lib().solon_layernorm_backward_workspace(rows, cols, partitions)


def solon_layernorm_backward(dy, x, mean, rstd, weight=None, partitions: int = 1, dx=None, dweight=None, dbias=None, param_grads: bool = True):
    """Gradients of layer norm.  Returns (dx, dweight, dbias); dweight and dbias are partitions x cols, row k summed over the
    rows of partition k (rows / partitions consecutive ones).  They may be views into the partition-gradient matrix
    (float32 or float64, as the plan's type), e.g. grads[:, a:a + cols].  param_grads=False: dx only."""
    import torch

    px, x_pitch = _matrix(x, "x")
    rows, cols = x.shape
    device, f32 = x.device, torch.float32
    pdy, dy_pitch = _matrix(dy, "dy", x)
    stream = _current_stream(device)
    if dx is None:
        dx = _empty_matrix(x)
        pdx, dx_pitch = dx.data_ptr(), cols
    else:
        pdx, dx_pitch = _matrix(dx, "dx", x)
    pw, _, code = _params(weight, None, cols, x)
    pdw = pdb = workspace = None
    grad_pitch, grad_code, n_bytes = cols, F32, 0
    if param_grads:
        like = dweight if dweight is not None else dbias
        if like is None:
            dweight, dbias = x.new_empty((2, partitions, cols), dtype=f32).unbind(0)
        elif dweight is None:
            dweight = torch.empty_strided(like.shape, like.stride(), dtype=like.dtype, device=device)
        elif dbias is None:
            dbias = torch.empty_strided(like.shape, like.stride(), dtype=like.dtype, device=device)
        if dweight.shape[0] != partitions or dweight.shape[-1] != cols or dweight.device != device:
            raise ValueError(f"dweight: expected {partitions} x {cols} on {device}, got {tuple(dweight.shape)} on {dweight.device}")
        pdw, grad_pitch = _matrix(dweight, "dweight")
        pdb, other_pitch = _matrix(dbias, "dbias", dweight)
        if grad_pitch != other_pitch:
            raise ValueError("dweight and dbias must have the same row pitch")
        grad_code = _dtype_code(dweight.dtype)
        n_bytes = _layernorm_workspace(rows, cols, partitions)
        if n_bytes > 0:
            workspace = x.new_empty(n_bytes // 4, dtype=f32)
    _check(lib().solon_layernorm_backward(pdy, dy_pitch, px, x_pitch, _dtype_code(x.dtype), pw, code, _vector(mean, "mean", rows, f32, device),
                                          _vector(rstd, "rstd", rows, f32, device), rows, cols, partitions, pdx, dx_pitch, pdw, pdb, grad_pitch,
                                          grad_code, None if workspace is None else workspace.data_ptr(), n_bytes, stream),
           "solon_layernorm_backward")
    return dx, dweight, dbias


class TokenLogprobs(NamedTuple):
    """What solon_token_logprobs returns; what was not asked for is None."""

    logp: object       # rows, float32: log probability of the target (None without targets)
    entropy: object    # rows, float32
    peak: object       # rows, float32: the largest logit (NaN if the row holds one)
    log_sum: object    # rows, float32: log sum e^(z - peak); log p = (z - peak) - log_sum
    top_ids: object    # rows x top_k, int64
    top_logp: object   # rows x top_k, float32


def solon_token_logprobs(logits, targets=None, top_k: int = 0) -> TokenLogprobs:
    """Log probabilities of the targets (int64; negative: none in this row) under the softmax of each row of logits
    (rows x vocabulary; float32, bfloat16 or float16), the rows' entropy and their top_k likeliest tokens.  Not recorded by
    autograd; the gradient is solon_token_logprobs_backward."""
    import torch

    pz, pitch = _matrix(logits, "logits")
    rows, vocab = logits.shape
    device = logits.device
    stream = _current_stream(device)
    f32 = torch.float32
    stats = logits.new_empty((4, rows), dtype=f32)
    base, row_bytes = stats.data_ptr(), 4 * rows
    top_ids = logits.new_empty((rows, top_k), dtype=torch.int64) if top_k > 0 else None
    top_logp = logits.new_empty((rows, top_k), dtype=f32) if top_k > 0 else None
    _check(lib().solon_token_logprobs(pz, pitch, _dtype_code(logits.dtype),
                                      None if targets is None else _vector(targets, "targets", rows, torch.int64, device), rows, vocab, top_k,
                                      None if targets is None else base, base + row_bytes, base + 2 * row_bytes, base + 3 * row_bytes,
                                      None if top_ids is None else top_ids.data_ptr(), None if top_logp is None else top_logp.data_ptr(), stream),
           "solon_token_logprobs")
    logp, entropy, peak, log_sum = stats.unbind(0)
    return TokenLogprobs(None if targets is None else logp, entropy, peak, log_sum, top_ids, top_logp)


def solon_token_logprobs_backward(logits, targets, peak, log_sum, grad_logp=None, entropy=None, grad_entropy=None, out=None):
    """Gradient of sum(grad_logp * logp + grad_entropy * entropy) with respect to the logits, in their type; `out` may be
    the logits themselves."""
    import torch

    pz, pitch = _matrix(logits, "logits")
    rows, vocab = logits.shape
    device = logits.device
    stream = _current_stream(device)
    if out is None:
        out = _empty_matrix(logits)
        po, out_pitch = out.data_ptr(), vocab
    else:
        po, out_pitch = _matrix(out, "out", logits)

    def row_vector(t, name):
        return None if t is None else _vector(t, name, rows, torch.float32, device)

    _check(lib().solon_token_logprobs_backward(pz, pitch, _dtype_code(logits.dtype),
                                               None if targets is None else _vector(targets, "targets", rows, torch.int64, device), rows, vocab,
                                               row_vector(peak, "peak"), row_vector(log_sum, "log_sum"),
                                               row_vector(entropy if grad_entropy is not None else None, "entropy"), row_vector(grad_logp, "grad_logp"),
                                               row_vector(grad_entropy, "grad_entropy"), po, out_pitch, stream),
           "solon_token_logprobs_backward")
    return out


class AdamW:
    """Owner of a solon_adamw*: AdamW over a list of float32 CUDA tensors, updated in place by step().

    bits: 32 or 8, the state's width.  weight_decay: one factor, or one per tensor.  copies: bfloat16 tensors of the same
    sizes (entries may be None) that every step fills with the rounded parameters.  Autograd does not see the updates.  state: (exp_avg, exp_avg_sq, base) as
    an earlier handle's `state` had it, taken over in place; by default zeros.  step: steps already applied to it."""

    def __init__(self, params, bits: int = 32, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay=0.0, seed: int = 0, step: int = 0, copies=None,
                 state=None):
        import torch

        self._h = None
        params = list(params)
        if not params:
            raise ValueError("no parameters")
        self.device = params[0].device
        _current_stream(self.device)
        n = len(params)
        for p in params:
            if not (p.is_cuda and p.is_contiguous() and p.dtype == torch.float32 and p.device == self.device):
                raise ValueError("parameters must be contiguous float32 CUDA tensors on one device")
        copies = [None] * n if copies is None else list(copies)
        decay = list(weight_decay) if hasattr(weight_decay, "__len__") else [float(weight_decay)] * n
        if len(copies) != n or len(decay) != n:
            raise ValueError("copies and weight_decay need an entry for each parameter")
        for p, c in zip(params, copies):
            if c is not None and not (c.is_contiguous() and c.dtype == torch.bfloat16 and c.device == self.device and c.numel() == p.numel()):
                raise ValueError("copies must be contiguous bfloat16 tensors of the parameters' sizes")
        self.params, self.copies, self.bits = params, copies, bits
        self.numel = [p.numel() for p in params]
        self.total = sum(self.numel)
        sizes = (c_int64 * n)(*self.numel)
        blocks = int(lib().solon_adamw_state_blocks(n, sizes))
        if blocks < 0:
            raise SolonError(blocks, "solon_adamw_state_blocks")
        if bits not in (8, 32):
            raise ValueError("bits must be 8 or 32")
        dtype = torch.float32 if bits == 32 else torch.uint8
        if state is None:
            state = (torch.zeros((blocks, 256), dtype=dtype, device=self.device), torch.zeros((blocks, 256), dtype=dtype, device=self.device),
                     None if bits == 32 else torch.zeros((blocks, 2), dtype=torch.int16, device=self.device))
        exp_avg, exp_avg_sq, base = state
        for t, want, kind in ((exp_avg, (blocks, 256), dtype), (exp_avg_sq, (blocks, 256), dtype), (base, (blocks, 2), torch.int16)):
            if t is base and bits == 32:
                continue
            if t is None or not (t.is_contiguous() and t.dtype == kind and t.device == self.device and tuple(t.shape) == want):
                raise ValueError(f"state: expected contiguous {kind} tensors of shape {want} on {self.device}")
        self.state = (exp_avg, exp_avg_sq, None if bits == 32 else base)
        self._norm = torch.zeros((), dtype=torch.float32, device=self.device)
        self._grads = None
        handle = c_void_p()
        torch.cuda.current_stream().synchronize()        # the state may just have been made
        _check(lib().solon_adamw_create(n, sizes, self._pointers(params), self._pointers(copies), (c_float * n)(*decay), bits,
                                        exp_avg.data_ptr() or 16, exp_avg_sq.data_ptr() or 16,
                                        None if bits == 32 else base.data_ptr() or 16,
                                        betas[0], betas[1], eps, seed, byref(handle)), "solon_adamw_create")
        self._h = handle
        if step:
            self.set_step(step)

    @staticmethod
    def _pointers(tensors):
        return (c_void_p * len(tensors))(*[None if t is None or t.numel() == 0 else t.data_ptr() for t in tensors])

    def close(self) -> None:
        if getattr(self, "_h", None):
            lib().solon_adamw_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def bind_grads(self, grads) -> None:
        """Gradients in tensors of their own (one type: float32, float64 or bfloat16), read in place by step(None, ...)."""
        grads = list(grads)
        if len(grads) != len(self.numel):
            raise ValueError("one gradient for each parameter")
        for g, n in zip(grads, self.numel):
            if not (g.is_cuda and g.is_contiguous() and g.device == self.device and g.numel() == n and g.dtype == grads[0].dtype):
                raise ValueError("gradients must be contiguous CUDA tensors of the parameters' sizes and of one type")
        _check(lib().solon_adamw_bind_grads(self._h, self._pointers(grads), _dtype_code(grads[0].dtype)), "solon_adamw_bind_grads")
        self._grads = grads

    def step(self, grad=None, lr: float = 1e-3, grad_scale: float = 1.0, max_norm: float = 0.0, plan=None):
        """One step on the current stream.  grad: the gradients of all parameters one after the other (the aggregate that
        decode returns; float32, float64 or bfloat16), or None for the bound ones.  max_norm > 0 clips the norm of
        grad_scale * grad and returns that norm (a device scalar, overwritten by the next step).  plan: the Plan whose
        decode made grad; the step changes nothing if that decode failed."""
        stream = _current_stream(self.device)
        code = F32
        if grad is not None:
            if not (grad.is_cuda and grad.is_contiguous() and grad.device == self.device and grad.numel() == self.total):
                raise ValueError(f"grad must be a contiguous CUDA tensor of {self.total} elements on {self.device}")
            code = _dtype_code(grad.dtype)
        if plan is not None and plan.stream_handle != stream:
            raise ValueError("the plan's calls go to another stream than the current one")
        _check(lib().solon_adamw_step(self._h, None if grad is None else grad.data_ptr() or 16, code, grad_scale, lr, max_norm,
                                      self._norm.data_ptr() if max_norm > 0 else None, None if plan is None else plan._h, stream), "solon_adamw_step")
        return self._norm if max_norm > 0 else None

    def set_step(self, step: int) -> None:
        _check(lib().solon_adamw_set_step(self._h, step), "solon_adamw_set_step")

    def steps(self) -> tuple[int, int]:
        """(steps applied, steps that changed nothing); synchronises."""
        applied, skipped = c_int64(0), c_int64(0)
        _check(lib().solon_adamw_get_steps(self._h, byref(applied), byref(skipped)), "solon_adamw_get_steps")
        return applied.value, skipped.value

    def moments(self):
        """(exp_avg, exp_avg_sq), blocks x 256: the state itself with 32 bits, what it stands for in bfloat16 with 8."""
        import torch

        if self.bits == 32:
            return self.state[0], self.state[1]
        out = [torch.empty(self.state[0].shape, dtype=torch.bfloat16, device=self.device) for _ in range(2)]
        stream = _current_stream(self.device)
        if out[0].numel():
            _check(lib().solon_adamw_moments(self._h, out[0].data_ptr(), out[1].data_ptr(), stream), "solon_adamw_moments")
        return out[0], out[1]

    def of_tensor(self, blocked, i: int):
        """The entries of parameter i in a blocks x 256 tensor (a state or what moments() returns), as a flat view."""
        first = sum(-(-n // 256) for n in self.numel[:i]) * 256
        return blocked.view(-1)[first:first + self.numel[i]]


# ------------------------------------------------------------------ plan


class Plan:
    """Owner of a solon_plan*.  Methods mirror the C calls; tensors are torch CUDA tensors (float32, contiguous)."""

    def __init__(self, P: int, s: int, m: int, r: int, d: int, seed: int = 0, stream=None, dtype: str = "f32"):
        import torch

        self._torch = torch
        if dtype not in ("f32", "f64"):
            raise ValueError("dtype must be 'f32' or 'f64'")
        self.dtype = dtype
        self.tdtype = torch.float64 if dtype == "f64" else torch.float32     # element type of gradients, coded vectors, aggregate
        handle = c_void_p()
        _check(lib().solon_plan_create_ex(P, s, m, r, d, seed, F64 if dtype == "f64" else F32, byref(handle)), "solon_plan_create_ex")
        self._h = handle
        self.P, self.s, self.m, self.r, self.d = P, s, m, r, d
        self.d_c = int(lib().solon_plan_dc(self._h))
        self.q = int(lib().solon_plan_num_groups(self._h))
        self.set_stream(stream if stream is not None else torch.cuda.current_stream())

    def close(self) -> None:
        if getattr(self, "_h", None):
            lib().solon_plan_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    # -- configuration
    def set_stream(self, stream) -> None:
        raw = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
        _check(lib().solon_plan_set_stream(self._h, c_void_p(raw)), "solon_plan_set_stream")
        self.stream_handle = int(raw)      # the cudaStream_t the plan's calls enqueue on

    def set_num_projections(self, K: int) -> None:
        _check(lib().solon_plan_set_num_projections(self._h, K), "solon_plan_set_num_projections")

    def reseed(self, seed: int) -> None:
        _check(lib().solon_plan_reseed(self._h, seed), "solon_plan_reseed")

    def set_fresh_projections(self, on: bool) -> None:
        """True: every decode projects with projection vectors no earlier decode used; False (default): the ones in memory
        are reused until reseed()."""
        _check(lib().solon_plan_set_fresh_projections(self._h, 1 if on else 0), "solon_plan_set_fresh_projections")

    def set_tolerance(self, tau: float) -> None:
        _check(lib().solon_plan_set_tolerance(self._h, tau), "solon_plan_set_tolerance")

    def set_early_locator(self, mode: int) -> None:
        """0: never start the locator on a partial projection; 1 (default): when the projection pass is long; 2: always;
        3: diagnostic, the locator's wait for the partial sums runs out (outcome 3), results unchanged."""
        _check(lib().solon_plan_set_early_locator(self._h, mode), "solon_plan_set_early_locator")

    def set_optimistic(self, mode: int) -> None:
        """0: the projection pass never recovers the aggregate itself; 1 (default): it does so, from the rows of the previous
        decode's recovery table, when in each of the last two decodes the table of the decode before would have served; 2: always.  The recovery
        kernel is skipped when the locator finds those rows trusted in this decode."""
        _check(lib().solon_plan_set_optimistic(self._h, mode), "solon_plan_set_optimistic")

    def optimistic_outcome(self) -> bool:
        """True if the recovery kernel of the most recent decode had nothing to do."""
        out = c_int(0)
        _check(lib().solon_plan_get_optimistic_outcome(self._h, byref(out)), "solon_plan_get_optimistic_outcome")
        return bool(out.value)

    def early_outcome(self) -> np.ndarray:
        """Per group: 0 no early run, 1 early answer confirmed, 2 not confirmed, 3 wait expired (last decode)."""
        out = np.zeros(self.q, dtype=np.int32)
        _check(lib().solon_plan_get_early_outcome(self._h, _dptr(out, c_int)), "solon_plan_get_early_outcome")
        return out

    def set_lsq_rows(self, rows: int) -> None:
        _check(lib().solon_plan_set_lsq_rows(self._h, rows), "solon_plan_set_lsq_rows")

    # -- queries
    @property
    def K(self) -> int:
        return int(lib().solon_plan_num_projections(self._h))

    def group_starts(self) -> list[int]:
        starts = [lib().solon_plan_group_start(self._h, g) for g in range(self.q)]
        return starts + [self.P]

    def group_sizes(self) -> list[int]:
        return [lib().solon_plan_group_size(self._h, g) for g in range(self.q)]

    def group_of(self, node: int) -> int:
        return lib().solon_plan_group_of(self._h, node)

    def node_scalars(self) -> np.ndarray:
        w = np.zeros(self.P, dtype=np.float64)
        _check(lib().solon_plan_get_node_scalars(self._h, _dptr(w, c_double)), "solon_plan_get_node_scalars")
        return w

    def projection_vectors(self) -> np.ndarray:
        f = np.zeros((self.K, self.d_c), dtype=np.float32)
        _check(lib().solon_plan_get_projection_vectors(self._h, _dptr(f, c_float)), "solon_plan_get_projection_vectors")
        return f

    def set_profiling(self, on: bool) -> None:
        _check(lib().solon_plan_set_profiling(self._h, 1 if on else 0), "solon_plan_set_profiling")

    def timings(self) -> dict:
        """Milliseconds of the most recent encode / projection / locator / recovery kernels (profiling on)."""
        ms = np.zeros(4, dtype=np.float32)
        _check(lib().solon_plan_get_timings(self._h, _dptr(ms, c_float)), "solon_plan_get_timings")
        return {"encode": float(ms[0]), "project": float(ms[1]), "locate": float(ms[2]), "recover": float(ms[3])}

    def kernel_launches(self) -> int:
        return int(lib().solon_plan_kernel_launches(self._h))

    # -- hot path
    def _dev(self, t, shape, dtype=None):
        dtype = dtype or self.tdtype
        if not (t.is_cuda and t.is_contiguous() and t.dtype == dtype and tuple(t.shape) == tuple(shape)):
            raise ValueError(f"expected a contiguous CUDA {dtype} tensor of shape {tuple(shape)}, got {tuple(t.shape)} {t.dtype}")
        return c_void_p(t.data_ptr())

    def encode(self, partition_grads, coded=None):
        torch = self._torch
        if coded is None:
            coded = torch.empty((self.P, self.d_c), dtype=self.tdtype, device=partition_grads.device)
        fn = lib().solon_encode_f64 if self.dtype == "f64" else lib().solon_encode
        _check(fn(self._h, self._dev(partition_grads, (self.P, self.d)), self._dev(coded, (self.P, self.d_c))),
               "solon_encode")
        return coded

    def decode(self, received, agg_grad=None, byz_mask=None):
        torch = self._torch
        if agg_grad is None:
            agg_grad = torch.empty(self.d, dtype=self.tdtype, device=received.device)
        if byz_mask is None:
            byz_mask = torch.empty(self.P, dtype=torch.uint8, device=received.device)
        fn = lib().solon_decode_f64 if self.dtype == "f64" else lib().solon_decode
        _check(fn(self._h, self._dev(received, (self.P, self.d_c)), self._dev(agg_grad, (self.d,)),
                                  self._dev(byz_mask, (self.P,), torch.uint8)), "solon_decode")
        return agg_grad, byz_mask

    def decode_project(self, received, rho, nu):
        """First half of the decode: rho (K x P) and nu (P), float64 device tensors, receive this plan's projections."""
        torch = self._torch
        _check(lib().solon_decode_project(self._h, self._dev(received, (self.P, self.d_c)),
                                          self._dev(rho, (self.K, self.P), torch.float64),
                                          self._dev(nu, (self.P,), torch.float64)), "solon_decode_project")
        return rho, nu

    def decode_finish(self, rho, nu, received, agg_grad=None, byz_mask=None):
        """Second half: locator and recovery from the given (summed) projections."""
        torch = self._torch
        if agg_grad is None:
            agg_grad = torch.empty(self.d, dtype=torch.float32, device=received.device)
        if byz_mask is None:
            byz_mask = torch.empty(self.P, dtype=torch.uint8, device=received.device)
        _check(lib().solon_decode_finish(self._h, self._dev(rho, (self.K, self.P), torch.float64),
                                         self._dev(nu, (self.P,), torch.float64),
                                         self._dev(received, (self.P, self.d_c)), self._dev(agg_grad, (self.d,)),
                                         self._dev(byz_mask, (self.P,), torch.uint8)), "solon_decode_finish")
        return agg_grad, byz_mask

    def overwrite_rows(self, matrix, nodes, rows):
        """matrix[nodes[i]] = rows[i] on the plan's stream (the adversary of a device-resident simulation).
        nodes: int32 CUDA tensor; rows: len(nodes) x d_c float32 CUDA tensor."""
        torch = self._torch
        n = int(nodes.numel())
        if n == 0:
            return matrix
        fn = lib().solon_overwrite_rows_f64 if self.dtype == "f64" else lib().solon_overwrite_rows
        _check(fn(self._h, self._dev(matrix, (self.P, self.d_c)), n, self._dev(nodes, (n,), torch.int32),
                                          self._dev(rows, (n, self.d_c))), "solon_overwrite_rows")
        return matrix

    def decode_status(self) -> int:
        return lib().solon_decode_status(self._h)

    def status(self) -> int:
        """solon_plan_status: OK, or ERR_INTERNAL once a bounded wait inside one of the plan's kernels has run out."""
        return lib().solon_plan_status(self._h)

    def lsq_grads(self, X, y, w, grads=None, rows: int | None = None):
        torch = self._torch
        if rows is not None:
            self.set_lsq_rows(rows)
        n = X.shape[0]
        if grads is None:
            grads = torch.empty((self.P, self.d), dtype=torch.float32, device=X.device)
        _check(lib().solon_lsq_grads(self._h, self._dev(X, (n, self.d)), self._dev(y, (n,)), self._dev(w, (self.d,)),
                                     self._dev(grads, (self.P, self.d))), "solon_lsq_grads")
        return grads

    def step_host(self, grads_host, byz_nodes, byz_rows_host, agg_host, mask_host) -> int:
        """solon_step_host: host tensors in (ideally pinned), host tensors out; returns the decode status."""
        torch = self._torch
        for t in (grads_host, agg_host, mask_host):
            if t.is_cuda or not t.is_contiguous():
                raise ValueError("solon_step_host takes contiguous host tensors")
        n_byz = len(byz_nodes)
        nodes = np.asarray(byz_nodes, dtype=np.int32)
        rows_ptr = c_void_p(byz_rows_host.data_ptr()) if n_byz else c_void_p(0)
        fn = lib().solon_step_host_f64 if self.dtype == "f64" else lib().solon_step_host
        return fn(self._h, c_void_p(grads_host.data_ptr()), n_byz,
                                     _dptr(nodes, c_int) if n_byz else None, rows_ptr,
                                     c_void_p(agg_host.data_ptr()), c_void_p(mask_host.data_ptr()))

    # -- introspection of the last decode
    def projections(self):
        rho = np.zeros((self.K, self.P), dtype=np.float64)
        nu = np.zeros(self.P, dtype=np.float64)
        _check(lib().solon_plan_get_projections(self._h, _dptr(rho, c_double), _dptr(nu, c_double)), "solon_plan_get_projections")
        return rho, nu

    def recovery(self):
        """Returns (n_rec[q], t[q], rec_rows (concatenated), coeff (sum n_rec x m))."""
        n_rec = np.zeros(self.q, dtype=np.int32)
        t = np.zeros(self.q, dtype=np.int32)
        rows = np.zeros(self.P, dtype=np.int32)
        coeff = np.zeros(self.P * self.m, dtype=np.float64)
        _check(lib().solon_plan_get_recovery(self._h, _dptr(n_rec, c_int), _dptr(t, c_int), _dptr(rows, c_int),
                                             _dptr(coeff, c_double)), "solon_plan_get_recovery")
        total = int(n_rec.sum())
        return n_rec, t, rows[:total].copy(), coeff[:total * self.m].reshape(total, self.m).copy()


# C-named aliases for callers that prefer the flat interface
def solon_plan_create(P, s, m, r, d, seed=0) -> Plan:
    return Plan(P, s, m, r, d, seed)


def solon_encode(plan: Plan, partition_grads, coded=None):
    return plan.encode(partition_grads, coded)


def solon_decode(plan: Plan, received, agg_grad=None, byz_mask=None):
    return plan.decode(received, agg_grad, byz_mask)


def solon_lsq_grads(plan: Plan, X, y, w, grads=None):
    return plan.lsq_grads(X, y, w, grads)
