"""ctypes binding of the C-ABI library (include/ll.h).

Argument marshalling only: every step of the path runs in the HIP kernels of libll.so.
PyTorch supplies device memory and the stream.  If the library has not been built
(`python -m paper_2604_06483_amd.build`) loading raises: there is no fallback.
"""
from __future__ import annotations

import ctypes
import functools
import os
from ctypes import POINTER, Structure, c_char_p, c_float, c_int, c_int32, c_int64, c_size_t, c_void_p

import torch

LL_OK, LL_EINVAL, LL_EWORKSPACE, LL_EHIP, LL_ESCRATCH = 0, -1, -2, -3, -4
LL_KMAX = 32
LL_STATIC_SCRATCH_BYTES = 64 << 20
LL_LIST_MAX = 64
LL_STATE_BLOCK = 256
LL_TENSOR_PARAM_BF16, LL_TENSOR_GRAD_BF16, LL_TENSOR_STATE_8BIT = 1, 2, 4
LL_PREFERENCE = {"logistic": 0, "hinge": 1, "square": 2}
LL_FLAG_TOPK_SOFTMAX = 1
LL_FLAG_REGISTER_STAGED = 2

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libll.so")
_lib = None


class ll_shape(Structure):
    _fields_ = [("N", c_int64), ("d", c_int32), ("V", c_int32)]


class LLError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        msg = lib().ll_error_string(code).decode()
        if code == LL_EHIP:
            msg += f" [hipError {lib().ll_last_hip_error()}]"
        super().__init__(f"{where}: {msg} ({code})")


class ll_capture_shape(Structure):
    _fields_ = [("L", c_int32), ("C", c_int32), ("T", c_int64), ("d", c_int32)]


class ll_tensor(Structure):
    _fields_ = [(n, c_void_p) for n in ("param", "grad", "m", "v", "m_scale", "v_scale", "copy")] + [("n", c_int64), ("flags", ctypes.c_uint32)]


class ll_adamw_options(Structure):
    _fields_ = [(n, ctypes.c_double) for n in ("rate", "beta1", "beta2", "eps", "decay", "max_norm")] + [("step", c_int64), ("seed", ctypes.c_uint32)]


_PROJECT_ARGS = [POINTER(ll_shape), c_void_p, c_size_t, c_void_p, c_void_p, c_void_p, c_float, c_int,
                 c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p]


def lib() -> ctypes.CDLL:
    """The loaded shared library with its prototypes set."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(f"{_LIB_PATH} is missing: build it with `python -m paper_2604_06483_amd.build`")
        L = ctypes.CDLL(_LIB_PATH)
        L.ll_workspace_bytes.argtypes = [POINTER(ll_shape), c_int]
        L.ll_workspace_bytes.restype = c_size_t
        L.ll_project.argtypes = _PROJECT_ARGS
        L.ll_project.restype = c_int
        L.ll_project_ex.argtypes = _PROJECT_ARGS[:6] + [c_void_p, ctypes.c_uint] + _PROJECT_ARGS[6:]
        L.ll_project_ex.restype = c_int
        L.ll_project_timed.argtypes = _PROJECT_ARGS + [POINTER(c_float)]
        L.ll_project_timed.restype = c_int
        L.ll_project_static.argtypes = _PROJECT_ARGS[:1] + _PROJECT_ARGS[3:]
        L.ll_project_static.restype = c_int
        L.ll_project_static_pass_rows.argtypes = [POINTER(ll_shape), c_int]
        L.ll_project_static_pass_rows.restype = c_int64
        L.ll_steer_workspace_bytes.argtypes = [c_int32]
        L.ll_steer_workspace_bytes.restype = c_size_t
        L.ll_steer_vector.argtypes = [c_void_p, c_int64, c_void_p, c_int64, c_int32, c_int, c_void_p,
                                      c_void_p, c_size_t, c_void_p]
        L.ll_steer_vector.restype = c_int
        L.ll_steer_inject.argtypes = [POINTER(ll_shape), c_void_p, c_void_p, c_float, c_void_p, c_float,
                                      c_void_p, c_void_p]
        L.ll_steer_inject.restype = c_int
        L.ll_steer_sweep_workspace_bytes.argtypes = [POINTER(ll_shape), c_int]
        L.ll_steer_sweep_workspace_bytes.restype = c_size_t
        L.ll_steer_sweep.argtypes = [POINTER(ll_shape), c_void_p, c_size_t, c_void_p, c_void_p, c_void_p, c_float,
                                     c_void_p, POINTER(c_float), c_int, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                     c_void_p]
        L.ll_steer_sweep.restype = c_int
        L.ll_steer_sweep_topk_workspace_bytes.argtypes = [POINTER(ll_shape), c_int, c_int]
        L.ll_steer_sweep_topk_workspace_bytes.restype = c_size_t
        L.ll_steer_sweep_topk.argtypes = [POINTER(ll_shape), c_void_p, c_size_t, c_void_p, c_void_p, c_void_p, c_float,
                                          c_void_p, POINTER(c_float), c_int, c_int, c_void_p, c_void_p, c_void_p, c_void_p,
                                          c_void_p, c_void_p]
        L.ll_steer_sweep_topk.restype = c_int
        L.ll_steer_inject_raw.argtypes = [POINTER(ll_shape), c_void_p, c_void_p, c_float, c_float, c_float, c_void_p, c_void_p]
        L.ll_steer_inject_raw.restype = c_int
        L.ll_capture_append.argtypes = [POINTER(ll_capture_shape), c_void_p, c_void_p, c_int64, c_int64, c_void_p]
        L.ll_capture_append.restype = c_int
        L.ll_block_norm.argtypes = [POINTER(ll_shape), c_void_p, c_void_p, c_void_p, c_int, c_float, c_void_p, c_void_p, c_float,
                                    c_void_p, c_void_p, c_void_p]
        L.ll_block_norm.restype = c_int
        L.ll_block_norm_grad_workspace_bytes.argtypes = [POINTER(ll_shape)]
        L.ll_block_norm_grad_workspace_bytes.restype = c_size_t
        L.ll_block_norm_grad.argtypes = [POINTER(ll_shape), c_void_p, c_size_t, c_void_p, c_void_p, c_void_p, c_int, c_float, c_void_p,
                                         c_void_p, c_float] + [c_void_p] * 8
        L.ll_block_norm_grad.restype = c_int
        for name in ("ll_logp", "ll_logp_grad", "ll_distill"):
            size = getattr(L, name + "_workspace_bytes")
            size.argtypes = [POINTER(ll_shape), c_int]
            size.restype = c_size_t
        lens = [POINTER(ll_shape), c_void_p, c_size_t, c_void_p, c_void_p, c_float, c_int, c_void_p]
        L.ll_logp.argtypes = lens + [c_void_p] * 4
        L.ll_logp.restype = c_int
        L.ll_logp_grad.argtypes = lens + [c_void_p] * 6
        L.ll_logp_grad.restype = c_int
        L.ll_distill.argtypes = lens + [c_void_p] * 5
        L.ll_distill.restype = c_int
        L.ll_policy_workspace_bytes.argtypes = [POINTER(ll_shape)]
        L.ll_policy_workspace_bytes.restype = c_size_t
        L.ll_policy.argtypes = lens[:6] + [c_void_p] * 5 + [c_float] * 3 + [c_void_p] * 4
        L.ll_policy.restype = c_int
        L.ll_preference_workspace_bytes.argtypes = [POINTER(ll_shape), c_int32]
        L.ll_preference_workspace_bytes.restype = c_size_t
        L.ll_preference.argtypes = lens[:6] + [c_void_p] * 2 + [c_int32] + [c_void_p] * 2 + [c_int] * 2 + [c_float] * 2 + [c_void_p] * 5
        L.ll_preference.restype = c_int
        L.ll_grad_norm_workspace_bytes.argtypes = [c_int32]
        L.ll_grad_norm_workspace_bytes.restype = c_size_t
        L.ll_grad_norm.argtypes = [c_void_p, c_int32,       # (addresses: a pointer made of a structure is a microsecond)
                                    c_void_p, c_size_t, c_void_p, c_void_p]
        L.ll_grad_norm.restype = c_int
        L.ll_adamw.argtypes = [c_void_p, c_int32] + [c_void_p] * 5
        L.ll_adamw.restype = c_int
        L.ll_error_string.argtypes = [c_int]
        L.ll_error_string.restype = c_char_p
        L.ll_last_hip_error.argtypes = []
        L.ll_last_hip_error.restype = c_int
        _lib = L
    return _lib


# A call of a decoding step (steer one row, append one token's slices) is two short kernels, and this module's own Python was what
# bounded it: 17.5 us for the pair with a c_void_p made for every pointer, a torch.cuda.Stream object for every call and reshapes
# that change nothing; 11.3 us without them (and 21.9 | 16.6 us for a steering direction and its injection).  With the argument structures of the last shapes
# kept, a tensor's shape asked for once and no calls for what an expression does, 10.4 | 9.4 us (host time, in turn; runs of one side differ by 0.1 to 1 us), and
# 10.3 | 9.5 where 200 row counts come in turn, more than are kept.
_Tensor, _BF16, _F32 = torch.Tensor, torch.bfloat16, torch.float32
_shape = functools.lru_cache(maxsize=64)(ll_shape)                     # (the library only reads them)
_capture_shape = functools.lru_cache(maxsize=64)(ll_capture_shape)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _check(t, dtype, name, shape=None):
    if not (isinstance(t, _Tensor) and t.is_cuda and t.dtype == dtype and t.is_contiguous()):
        raise TypeError(f"{name}: need a contiguous {dtype} tensor on the GPU")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")


# torch.cuda.current_stream().cuda_stream without the object: torch's own, but not public, so only where they are there
_raw_stream, _device = (getattr(torch._C, n, None) for n in ("_cuda_getCurrentRawStream", "_cuda_getDevice"))


def _stream(stream):
    if stream is None and _raw_stream is not None and _device is not None:
        return _raw_stream(_device())
    return (torch.cuda.current_stream() if stream is None else stream).cuda_stream


def _rows(t, d, stream=None):
    """t as [rows, d]; a matrix of that width as it is (a reshape of it would be the same tensor in another object).

    A batch whose strides do not allow that is copied, and the copy has to be the work and the memory of the stream that the call goes to:
    made on another, the kernel would not wait for it, and its memory could be handed out again while the kernel still reads it."""
    size = t.shape
    if len(size) == 2 and size[1] == d:
        return t
    if stream is None or t.is_contiguous():
        return t.reshape(-1, d)
    with torch.cuda.stream(stream):
        return t.reshape(-1, d)


def _empty(size, dtype, device, stream):
    """A tensor that a call on `stream` writes: of that stream's own memory, which no earlier work of another stream still uses, and not
    given back to it before what the current stream has queued until the tensor is dropped."""
    if stream is None:
        return torch.empty(size, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        t = torch.empty(size, dtype=dtype, device=device)
    t.record_stream(torch.cuda.current_stream(device))
    return t


def _like(t, stream):
    return torch.empty_like(t) if stream is None else _empty(t.shape, t.dtype, t.device, stream)   # (1.2 us of host time against 1.75)


def _scratch(nbytes, device, stream):
    """A workspace of this call's own: released when the call returns, while the kernels may still be queued."""
    return _empty((max(int(nbytes), 256),), torch.uint8, device, stream)


def ll_workspace_bytes(N: int, d: int, V: int, k: int) -> int:
    return int(lib().ll_workspace_bytes(ll_shape(N, d, V), k))


def ll_steer_workspace_bytes(d: int) -> int:
    return int(lib().ll_steer_workspace_bytes(d))


def ll_project(hidden, gamma, W_U, eps, k, target_ids=None, *, workspace=None, stream=None, out=None, timed=False,
               bias=None, topk_softmax=False, register_staged=False):
    """hidden [..., d] bf16, gamma [d] bf16 or None, W_U [V, d] bf16, target_ids [N] int32 or None.
    bias [V] fp32 (the b of Eq. 1), topk_softmax (probabilities over the k selected logits only, the paper's
    own output format) and register_staged (the kernel with the norm inside its A-tile load) go through
    ll_project_ex.

    Returns (topk_ids [N,k] int32, topk_p [N,k] fp32, target_logp [N] fp32 or None, entropy [N] fp32),
    plus the three phase times in ms when timed=True (that variant synchronises the stream).
    """
    d = hidden.shape[-1]
    h2 = _rows(hidden, d, stream)
    N = h2.shape[0]
    V = W_U.shape[0]
    _check(h2, torch.bfloat16, "hidden")
    _check(W_U, torch.bfloat16, "W_U", (V, d))
    if gamma is not None:
        _check(gamma, torch.bfloat16, "gamma", (d,))
    if target_ids is not None:
        _check(target_ids, torch.int32, "target_ids", (N,))
    shape = ll_shape(N, d, V)
    need = int(lib().ll_workspace_bytes(shape, k))
    if workspace is None:
        workspace = _scratch(need, hidden.device, stream)
    dev = hidden.device
    if out is None:
        ids = _empty((N, k), torch.int32, dev, stream)
        p = _empty((N, k), torch.float32, dev, stream)
        logp = _empty((N,), torch.float32, dev, stream) if target_ids is not None else None
        ent = _empty((N,), torch.float32, dev, stream)
    else:
        ids, p, logp, ent = out
    args = [shape, _ptr(workspace), workspace.numel() * workspace.element_size(), _ptr(h2), _ptr(gamma), _ptr(W_U),
            float(eps), int(k), _ptr(target_ids), _ptr(ids), _ptr(p), _ptr(logp), _ptr(ent), _stream(stream)]
    if bias is not None or topk_softmax or register_staged:
        if timed:
            raise ValueError("the timed variant has no bias / top-k-softmax / kernel-choice form")
        if bias is not None:
            _check(bias, torch.float32, "bias", (V,))
        flags = (LL_FLAG_TOPK_SOFTMAX if topk_softmax else 0) | (LL_FLAG_REGISTER_STAGED if register_staged else 0)
        rc = lib().ll_project_ex(*args[:6], _ptr(bias), flags, *args[6:])
        if rc != LL_OK:
            raise LLError(rc, "ll_project_ex")
        return ids, p, logp, ent
    if timed:
        ms = (c_float * 3)()
        rc = lib().ll_project_timed(*args, ms)
        if rc != LL_OK:
            raise LLError(rc, "ll_project_timed")
        return ids, p, logp, ent, [float(x) for x in ms]
    rc = lib().ll_project(*args)
    if rc != LL_OK:
        raise LLError(rc, "ll_project")
    return ids, p, logp, ent


def ll_project_static_pass_rows(N: int, d: int, V: int, k: int) -> int:
    return int(lib().ll_project_static_pass_rows(ll_shape(N, d, V), k))


def ll_project_static(hidden, gamma, W_U, eps, k, target_ids=None, *, stream=None, out=None):
    """ll_project without a workspace: the library's own static device buffer holds the partial results, and the
    call allocates nothing (pass `out` to keep this wrapper from allocating the result tensors).  Calls that may
    overlap on one GPU race on that buffer.  Same results as ll_project."""
    d = hidden.shape[-1]
    h2 = _rows(hidden, d, stream)
    N = h2.shape[0]
    V = W_U.shape[0]
    _check(h2, torch.bfloat16, "hidden")
    _check(W_U, torch.bfloat16, "W_U", (V, d))
    if gamma is not None:
        _check(gamma, torch.bfloat16, "gamma", (d,))
    if target_ids is not None:
        _check(target_ids, torch.int32, "target_ids", (N,))
    dev = hidden.device
    if out is None:
        ids = _empty((N, k), torch.int32, dev, stream)
        p = _empty((N, k), torch.float32, dev, stream)
        logp = _empty((N,), torch.float32, dev, stream) if target_ids is not None else None
        ent = _empty((N,), torch.float32, dev, stream)
    else:
        ids, p, logp, ent = out
    rc = lib().ll_project_static(ll_shape(N, d, V), _ptr(h2), _ptr(gamma), _ptr(W_U), float(eps), int(k), _ptr(target_ids),
                                 _ptr(ids), _ptr(p), _ptr(logp), _ptr(ent), _stream(stream))
    if rc != LL_OK:
        raise LLError(rc, "ll_project_static")
    return ids, p, logp, ent


def ll_steer_vector(base, target, normalize=True, *, workspace=None, stream=None, out=None):
    """base [Nb, d], target [Nt, d] bf16 -> v [d] fp32 (paper Eq. 2)."""
    _check(base, _BF16, "base")
    _check(target, _BF16, "target")
    b_size, t_size = base.shape, target.shape
    d = b_size[-1]
    if t_size[-1] != d or len(b_size) != 2 or len(t_size) != 2:
        raise ValueError("base and target must be [rows, d] with the same d")
    v = _empty((d,), torch.float32, base.device, stream) if out is None else out
    wsb = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = (_lib or lib()).ll_steer_vector(base.data_ptr(), b_size[0], target.data_ptr(), t_size[0], d, 1 if normalize else 0,
                                         v.data_ptr(), _ptr(workspace), wsb, _stream(stream))
    if rc != LL_OK:
        raise LLError(rc, "ll_steer_vector")
    return v


def ll_steer_inject(hidden, gamma, eps, v, alpha, *, stream=None, out=None):
    """bf16(RMSNorm(hidden) + alpha v), same shape as hidden (paper Eq. 3, post-norm)."""
    size = hidden.shape
    d = size[-1]
    h2 = hidden if len(size) == 2 else hidden.reshape(-1, d) if stream is None else _rows(hidden, d, stream)
    _check(h2, _BF16, "hidden")
    _check(gamma, _BF16, "gamma", (d,))
    _check(v, _F32, "v", (d,))
    o = _rows(out, d) if out is not None else torch.empty_like(h2) if stream is None else _like(h2, stream)
    rc = (_lib or lib()).ll_steer_inject(_shape(h2.shape[0], d, 0), h2.data_ptr(), gamma.data_ptr(), float(eps), v.data_ptr(), float(alpha),
                                         o.data_ptr(), _stream(stream))
    if rc != LL_OK:
        raise LLError(rc, "ll_steer_inject")
    return o if o.shape == size else o.reshape(size)


LL_SWEEP_MAX = 9
LL_SWEEP_KMAX = 4


def ll_steer_sweep_workspace_bytes(N: int, d: int, V: int, n_alpha: int, k: int = 1) -> int:
    if k == 1:
        return int(lib().ll_steer_sweep_workspace_bytes(ll_shape(N, d, V), n_alpha))
    return int(lib().ll_steer_sweep_topk_workspace_bytes(ll_shape(N, d, V), n_alpha, k))


def ll_steer_sweep(hidden, gamma, W_U, eps, v, alphas, target_ids=None, *, k=None, workspace=None, stream=None):
    """Lens read-out of the steered rows RMSNorm(hidden) + alpha v for every alpha of the list in one pass over
    W_U (paper Eq. 3 / Sec. 3.4).  v [d] fp32 on the GPU, alphas a sequence of at most LL_SWEEP_MAX floats.

    Returns (top1_ids [A,N] int32, top1_p [A,N] fp32, target_logp [A,N] fp32 or None, entropy [A,N] fp32);
    with k given (1..LL_SWEEP_KMAX, through ll_steer_sweep_topk) the first two are [A,N,k] lists.
    """
    d = hidden.shape[-1]
    h2 = _rows(hidden, d, stream)
    N = h2.shape[0]
    V = W_U.shape[0]
    A = len(alphas)
    _check(h2, torch.bfloat16, "hidden")
    _check(W_U, torch.bfloat16, "W_U", (V, d))
    _check(v, torch.float32, "v", (d,))
    if gamma is not None:
        _check(gamma, torch.bfloat16, "gamma", (d,))
    if target_ids is not None:
        _check(target_ids, torch.int32, "target_ids", (N,))
    shape = ll_shape(N, d, V)
    need = ll_steer_sweep_workspace_bytes(N, d, V, A, 1 if k is None else int(k))
    if workspace is None:
        workspace = _scratch(need, hidden.device, stream)
    dev = hidden.device
    ids = _empty((A, N) if k is None else (A, N, int(k)), torch.int32, dev, stream)
    p = _empty((A, N) if k is None else (A, N, int(k)), torch.float32, dev, stream)
    logp = _empty((A, N), torch.float32, dev, stream) if target_ids is not None else None
    ent = _empty((A, N), torch.float32, dev, stream)
    al = (c_float * max(A, 1))(*[float(x) for x in alphas])
    if k is None:
        rc = lib().ll_steer_sweep(shape, _ptr(workspace), workspace.numel() * workspace.element_size(), _ptr(h2), _ptr(gamma),
                                  _ptr(W_U), float(eps), _ptr(v), al, A, _ptr(target_ids), _ptr(ids), _ptr(p), _ptr(logp),
                                  _ptr(ent), _stream(stream))
    else:
        rc = lib().ll_steer_sweep_topk(shape, _ptr(workspace), workspace.numel() * workspace.element_size(), _ptr(h2),
                                       _ptr(gamma), _ptr(W_U), float(eps), _ptr(v), al, A, int(k), _ptr(target_ids), _ptr(ids),
                                       _ptr(p), _ptr(logp), _ptr(ent), _stream(stream))
    if rc != LL_OK:
        raise LLError(rc, "ll_steer_sweep" if k is None else "ll_steer_sweep_topk")
    return ids, p, logp, ent


def ll_steer_inject_raw(hidden, v, alpha, layer_scale=1.0, clip_ratio=0.0, *, stream=None, out=None):
    """bf16(hidden + beta v) with beta = alpha * layer_scale clipped to clip_ratio * ||row||_2 (paper Sec. 3.4,
    in-model injection with its two safeguards); same shape as hidden."""
    size = hidden.shape
    d = size[-1]
    h2 = hidden if len(size) == 2 else hidden.reshape(-1, d) if stream is None else _rows(hidden, d, stream)
    _check(h2, _BF16, "hidden")
    _check(v, _F32, "v", (d,))
    o = _rows(out, d) if out is not None else torch.empty_like(h2) if stream is None else _like(h2, stream)
    rc = (_lib or lib()).ll_steer_inject_raw(_shape(h2.shape[0], d, 0), h2.data_ptr(), v.data_ptr(), float(alpha), float(layer_scale),
                                             float(clip_ratio), o.data_ptr(), _stream(stream))
    if rc != LL_OK:
        raise LLError(rc, "ll_steer_inject_raw")
    return o if o.shape == size else o.reshape(size)


def ll_capture_append(store, slices, t0, *, stream=None):
    """store [L, C, T, d] bf16, slices [L*C, n_tok, d] bf16: writes tokens t0 .. t0+n_tok-1 of every trajectory
    (paper Sec. 3.1 Stage 2).  store.reshape(-1, d) is then what ll_project takes."""
    _check(store, _BF16, "store")
    size = store.shape
    if len(size) != 4:
        raise ValueError("store: need [L, C, T, d]")
    L, C, T, d = size
    _check(slices, _BF16, "slices")
    got = slices.shape
    if len(got) != 3 or got[0] != L * C or got[2] != d:
        raise ValueError(f"slices: shape {tuple(got)}, expected ({L * C}, n_tok, {d})")
    rc = (_lib or lib()).ll_capture_append(_capture_shape(L, C, T, d), store.data_ptr(), slices.data_ptr(), int(t0), got[1], _stream(stream))
    if rc != LL_OK:
        raise LLError(rc, "ll_capture_append")


def _gate(gate, N, d, stream):
    """The gate, [d] for all rows or [N, d], and whether it is a row's own."""
    if gate is None:
        return None, 0
    g = _rows(gate, d, stream) if gate.dim() > 2 and gate.shape[-1] == d else gate
    _check(g, _BF16, "gate", (d,) if g.dim() == 1 else (N, d))
    return g, g.dim() - 1


def _workspace(workspace, need, device, stream):
    if workspace is None:
        return _scratch(need(), device, stream)
    if not (isinstance(workspace, _Tensor) and workspace.is_cuda and workspace.is_contiguous()):
        raise TypeError("workspace: need a contiguous tensor on the GPU")
    return workspace


def ll_block_norm(hidden, y, gamma, eps, *, gate=None, scale=1.0, gamma_y=None, stream=None, out=None):
    """The residual and the norms around a block: x = hidden + scale gate u, u = y or gamma_y y / rms(y).

    hidden, y [..., d] bf16, gamma [d] bf16, gate None, [d] or, a row's own, [..., d] bf16, gamma_y None or [d] bf16.
    Returns (x, gamma x / rms(x)), both bf16 in hidden's shape (`out`: two tensors to hold them).
    """
    d = hidden.shape[-1]
    h2, y2 = _rows(hidden, d, stream), _rows(y, d, stream)
    N = h2.shape[0]
    _check(h2, _BF16, "hidden")
    _check(y2, _BF16, "y", (N, d))
    _check(gamma, _BF16, "gamma", (d,))
    if gamma_y is not None:
        _check(gamma_y, _BF16, "gamma_y", (d,))
    if out is None:
        x, n = _like(h2, stream), _like(h2, stream)
    else:
        x, n = out
        for t, name in ((x, "out[0]"), (n, "out[1]")):
            _check(t, _BF16, name)
            if t.numel() != N * d:
                raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(hidden.shape)}")
    k2, gate_rows = _gate(gate, N, d, stream)
    rc = (_lib or lib()).ll_block_norm(_shape(N, d, 0), h2.data_ptr(), y2.data_ptr(), _ptr(k2), gate_rows, float(scale),
                                       _ptr(gamma_y), gamma.data_ptr(), float(eps), x.data_ptr(), n.data_ptr(), _stream(stream))
    if rc != LL_OK:
        raise LLError(rc, "ll_block_norm")
    return (x, n) if x.shape == hidden.shape else (x.reshape(hidden.shape), n.reshape(hidden.shape))


def ll_block_norm_grad_workspace_bytes(N: int, d: int) -> int:
    return int(lib().ll_block_norm_grad_workspace_bytes(ll_shape(N, d, 0)))


def ll_block_norm_grad(hidden, y, gamma, eps, g_hidden, g_normed, *, gate=None, scale=1.0, gamma_y=None, workspace=None, stream=None):
    """Gradient of ll_block_norm: from its inputs, g_hidden (of x; None: zero) and g_normed, bf16 in hidden's shape.

    Returns (d_hidden, d_y, d_gate, d_gamma_y, d_gamma): bf16 in hidden's shape, d_gate as the gate is (fp32 [d] or bf16 [..., d]; None without one),
    fp32 [d] (d_gamma_y None without gamma_y).
    """
    size, d = hidden.shape, hidden.shape[-1]
    h2, y2, gn = _rows(hidden, d, stream), _rows(y, d, stream), _rows(g_normed, d, stream)
    gh = None if g_hidden is None else _rows(g_hidden, d, stream)
    N = h2.shape[0]
    _check(h2, _BF16, "hidden")
    _check(y2, _BF16, "y", (N, d))
    _check(gn, _BF16, "g_normed", (N, d))
    if gh is not None:
        _check(gh, _BF16, "g_hidden", (N, d))
    _check(gamma, _BF16, "gamma", (d,))
    if gamma_y is not None:
        _check(gamma_y, _BF16, "gamma_y", (d,))
    k2, gate_rows = _gate(gate, N, d, stream)
    dev = hidden.device
    dh, dy = _like(h2, stream), _like(h2, stream)
    dk = None if gate is None else _like(k2, stream) if gate_rows else _empty((d,), _F32, dev, stream)
    dgy = None if gamma_y is None else _empty((d,), _F32, dev, stream)
    dg = _empty((d,), _F32, dev, stream)
    ws = _workspace(workspace, lambda: ll_block_norm_grad_workspace_bytes(N, d), dev, stream)
    rc = (_lib or lib()).ll_block_norm_grad(_shape(N, d, 0), ws.data_ptr(), ws.numel() * ws.element_size(), h2.data_ptr(), y2.data_ptr(),
                                            _ptr(k2), gate_rows, float(scale), _ptr(gamma_y), gamma.data_ptr(), float(eps), _ptr(gh),
                                            gn.data_ptr(), dh.data_ptr(), dy.data_ptr(), _ptr(dk), _ptr(dgy), dg.data_ptr(), _stream(stream))
    if rc != LL_OK:
        raise LLError(rc, "ll_block_norm_grad")
    if gate_rows and dk.shape != gate.shape:
        dk = dk.reshape(gate.shape)
    return dh if dh.shape == size else dh.reshape(size), dy if dy.shape == size else dy.reshape(size), dk, dgy, dg


def ll_logp_workspace_bytes(N: int, d: int, V: int, k: int) -> int:
    return int(lib().ll_logp_workspace_bytes(ll_shape(N, d, V), k))


def ll_logp_grad_workspace_bytes(N: int, d: int, V: int, k: int) -> int:
    return int(lib().ll_logp_grad_workspace_bytes(ll_shape(N, d, V), k))


def ll_distill_workspace_bytes(N: int, d: int, V: int, k: int) -> int:
    return int(lib().ll_distill_workspace_bytes(ll_shape(N, d, V), k))


def _lens_rows(rows, W_U, ids, name, stream):
    """Rows as [N, d], the list as [N, k], and (N, d, V, k)."""
    d = rows.shape[-1]
    r2 = _rows(rows, d, stream)
    N, V = r2.shape[0], W_U.shape[0]
    _check(r2, _BF16, "rows")
    _check(W_U, _BF16, "W_U", (V, d))
    k = ids.shape[-1] if ids.dim() > 1 else 1
    i2 = ids if ids.dim() == 2 else _rows(ids, k, stream)
    _check(i2, torch.int32, name, (N, k))
    return r2, i2, N, d, V, k


def ll_logp(rows, W_U, ids, *, temperature=1.0, workspace=None, stream=None):
    """Log-probabilities of listed tokens: rows [..., d] bf16 (normalised), W_U [V, d] bf16, ids [N, k] int32 (or [N], k = 1).

    Returns (logp [N, k], logsumexp [N], entropy [N]), fp32.
    """
    r2, i2, N, d, V, k = _lens_rows(rows, W_U, ids, "ids", stream)
    dev = rows.device
    logp, lse, ent = _empty((N, k), _F32, dev, stream), _empty((N,), _F32, dev, stream), _empty((N,), _F32, dev, stream)
    ws = _workspace(workspace, lambda: ll_logp_workspace_bytes(N, d, V, k), dev, stream)
    rc = (_lib or lib()).ll_logp(_shape(N, d, V), ws.data_ptr(), ws.numel() * ws.element_size(), r2.data_ptr(), W_U.data_ptr(),
                                 float(temperature), k, i2.data_ptr(), logp.data_ptr(), lse.data_ptr(), ent.data_ptr(), _stream(stream))
    if rc != LL_OK:
        raise LLError(rc, "ll_logp")
    return logp, lse, ent


def ll_logp_grad(rows, W_U, ids, lse, entropy, g_logp, g_entropy=None, *, temperature=1.0, workspace=None, stream=None):
    """Gradient of ll_logp to its rows, from its own lse and entropy (None without g_entropy), g_logp [N, k] and g_entropy [N] or None.

    Returns it in bf16 in the rows' shape.
    """
    r2, i2, N, d, V, k = _lens_rows(rows, W_U, ids, "ids", stream)
    g2 = g_logp if g_logp.dim() == 2 else _rows(g_logp, k, stream)
    _check(g2, _F32, "g_logp", (N, k))
    _check(lse, _F32, "lse", (N,))
    for t, name in ((entropy, "entropy"), (g_entropy, "g_entropy")):
        if t is not None:
            _check(t, _F32, name, (N,))
    out = _like(r2, stream)
    ws = _workspace(workspace, lambda: ll_logp_grad_workspace_bytes(N, d, V, k), rows.device, stream)
    rc = (_lib or lib()).ll_logp_grad(_shape(N, d, V), ws.data_ptr(), ws.numel() * ws.element_size(), r2.data_ptr(), W_U.data_ptr(),
                                      float(temperature), k, i2.data_ptr(), lse.data_ptr(), _ptr(entropy), g2.data_ptr(), _ptr(g_entropy),
                                      out.data_ptr(), _stream(stream))
    if rc != LL_OK:
        raise LLError(rc, "ll_logp_grad")
    return out if out.shape == rows.shape else out.reshape(rows.shape)


def ll_distill(rows, W_U, teacher_ids, teacher_scores, *, temperature=1.0, weight=None, grad=True, workspace=None, stream=None):
    """Distillation from a teacher's top tokens: teacher_ids [N, k] int32 (an id outside the vocabulary: no entry), teacher_scores [N, k]
    fp32 (logits or log-probabilities, as the logarithm of ll_project's lists), weight [N] fp32 or None (1).

    Returns (loss [N] fp32, gradient of weight . loss in bf16 in the rows' shape, or None with grad=False).
    """
    r2, i2, N, d, V, k = _lens_rows(rows, W_U, teacher_ids, "teacher_ids", stream)
    s2 = teacher_scores if teacher_scores.dim() == 2 else _rows(teacher_scores, k, stream)
    _check(s2, _F32, "teacher_scores", (N, k))
    if weight is not None:
        _check(weight, _F32, "weight", (N,))
    loss = _empty((N,), _F32, rows.device, stream)
    out = _like(r2, stream) if grad else None
    ws = _workspace(workspace, lambda: (ll_distill_workspace_bytes if grad else ll_logp_workspace_bytes)(N, d, V, k), rows.device, stream)
    rc = (_lib or lib()).ll_distill(_shape(N, d, V), ws.data_ptr(), ws.numel() * ws.element_size(), r2.data_ptr(), W_U.data_ptr(),
                                    float(temperature), k, i2.data_ptr(), s2.data_ptr(), _ptr(weight), loss.data_ptr(), _ptr(out),
                                    _stream(stream))
    if rc != LL_OK:
        raise LLError(rc, "ll_distill")
    return loss, out if out is None or out.shape == rows.shape else out.reshape(rows.shape)


def ll_policy_workspace_bytes(N: int, d: int, V: int) -> int:
    return int(lib().ll_policy_workspace_bytes(ll_shape(N, d, V)))


def ll_preference_workspace_bytes(N: int, d: int, V: int, pairs: int) -> int:
    return int(lib().ll_preference_workspace_bytes(ll_shape(N, d, V), pairs))


def _here(device, stream, *others):
    """All tensors on one device, and that the one that the call goes to: a kernel would read the others' addresses as its own."""
    for t in others:
        if t is not None and t.device != device:
            raise ValueError(f"tensors on {device} and on {t.device}")
    index = (None if _device is None else _device()) if stream is None else stream.device.index
    if index is not None and device.index is not None and index != device.index:
        raise ValueError(f"the tensors are on {device}, the call goes to device {index}")


def _each(t, dtype, name, N, stream):
    """One value a row, in the rows' own leading shape or flat."""
    if t is None:
        return None
    if isinstance(t, _Tensor) and t.dim() != 1:
        t = _rows(t, 1, stream).reshape(-1)
    _check(t, dtype, name, (N,))
    return t


def _answer_rows(rows, W_U, ids, stream):
    d = rows.shape[-1]
    r2 = _rows(rows, d, stream)
    N, V = r2.shape[0], W_U.shape[0]
    _check(r2, _BF16, "rows")
    _check(W_U, _BF16, "W_U", (V, d))
    return r2, _each(ids, torch.int32, "ids", N, stream), N, d, V


def ll_policy(rows, W_U, ids, advantage, old_logp=None, *, ref_logp=None, weight=None, clip=(0.2, 0.2), kl=0.0, temperature=1.0, grad=True,
              workspace=None, stream=None):
    """Clipped policy loss with a KL term over sampled tokens: rows [..., d] bf16 (normalised), W_U [V, d] bf16, ids int32, advantage, old_logp
    (None: on policy), ref_logp (None: only with kl 0) and weight (None: 1) fp32, one a row; clip: how far the ratio may fall below and rise above 1.

    Returns (loss [N] fp32, the tokens' log-probabilities [N] fp32, gradient of weight . loss in bf16 in the rows' shape, or None with grad=False).
    """
    r2, i2, N, d, V = _answer_rows(rows, W_U, ids, stream)
    A, old, ref, w = (_each(t, _F32, name, N, stream) for t, name in ((advantage, "advantage"), (old_logp, "old_logp"), (ref_logp, "ref_logp"), (weight, "weight")))
    dev = rows.device
    _here(dev, stream, W_U, i2, A, old, ref, w, workspace)
    loss, logp = _empty((N,), _F32, dev, stream), _empty((N,), _F32, dev, stream)
    out = _like(r2, stream) if grad else None
    ws = _workspace(workspace, lambda: ll_policy_workspace_bytes(N, d, V) if grad else ll_logp_workspace_bytes(N, d, V, 1), dev, stream)
    rc = (_lib or lib()).ll_policy(_shape(N, d, V), ws.data_ptr(), ws.numel() * ws.element_size(), r2.data_ptr(), W_U.data_ptr(), float(temperature),
                                   i2.data_ptr(), _ptr(A), _ptr(old), _ptr(ref), _ptr(w), float(clip[0]), float(clip[1]), float(kl),
                                   loss.data_ptr(), logp.data_ptr(), _ptr(out), _stream(stream))
    if rc != LL_OK:
        raise LLError(rc, "ll_policy")
    return loss, logp, out if out is None or out.shape == rows.shape else out.reshape(rows.shape)


def ll_preference(rows, W_U, ids, offsets, *, ref_logp=None, weight=None, beta=0.1, smoothing=0.0, form="logistic", mean=False, temperature=1.0,
                  grad=True, workspace=None, stream=None):
    """Preference loss over pairs of answers: rows [..., d] bf16 (normalised), W_U [V, d] bf16, ids int32 and ref_logp fp32 (None: 0), one a row;
    offsets int32 [2 pairs + 1], on the GPU: where the sequences begin and end, the preferred one of a pair first; weight fp32 [pairs] or None (1).
    form: "logistic", "hinge" or "square"; mean: scores a token instead of a sequence.

    Returns (loss [pairs] fp32, scores [pairs, 2] fp32, the tokens' log-probabilities [N] fp32, gradient of weight . loss in bf16 in the rows'
    shape, or None with grad=False).
    """
    if form not in LL_PREFERENCE:
        raise ValueError(f"form: {form!r}, expected one of {sorted(LL_PREFERENCE)}")
    r2, i2, N, d, V = _answer_rows(rows, W_U, ids, stream)
    _check(offsets, torch.int32, "offsets")
    if offsets.dim() != 1 or offsets.shape[0] % 2 != 1:
        raise ValueError(f"offsets: shape {tuple(offsets.shape)}, expected (2 pairs + 1,)")
    P = offsets.shape[0] // 2
    ref, w = _each(ref_logp, _F32, "ref_logp", N, stream), _each(weight, _F32, "weight", P, stream)
    dev = rows.device
    _here(dev, stream, W_U, i2, offsets, ref, w, workspace)
    loss, score, logp = _empty((P,), _F32, dev, stream), _empty((P, 2), _F32, dev, stream), _empty((N,), _F32, dev, stream)
    out = _like(r2, stream) if grad else None
    ws = _workspace(workspace, lambda: ll_preference_workspace_bytes(N, d, V, P) if grad else ll_logp_workspace_bytes(N, d, V, 1), dev, stream)
    rc = (_lib or lib()).ll_preference(_shape(N, d, V), ws.data_ptr(), ws.numel() * ws.element_size(), r2.data_ptr(), W_U.data_ptr(),
                                       float(temperature), i2.data_ptr(), offsets.data_ptr(), P, _ptr(ref), _ptr(w), LL_PREFERENCE[form],
                                       1 if mean else 0, float(beta), float(smoothing), loss.data_ptr(), score.data_ptr(), logp.data_ptr(),
                                       _ptr(out), _stream(stream))
    if rc != LL_OK:
        raise LLError(rc, "ll_preference")
    return loss, score, logp, out if out is None or out.shape == rows.shape else out.reshape(rows.shape)


class TensorList:
    """The tensors that a step is about, as ll_grad_norm and ll_adamw take them, checked and marshalled once: `grads` alone for the norm; for a
    step also `params`, `m` and `v` (fp32; or m in float8_e4m3fn and v in float8_e5m2 with fp32 `m_scale` and `v_scale`, one for LL_STATE_BLOCK
    elements) and, where fp32 parameters have one, a bf16 copy each (`copies`; None: none).  Their memory is kept, and worked on in place: of a
    tensor that is given other memory later (by `.data =`, say) it is still the old.  All on one device.
    """

    def __init__(self, grads, params=None, m=None, v=None, m_scale=None, v_scale=None, copies=None):
        kinds = {"params": params, "m": m, "v": v, "m_scale": m_scale, "v_scale": v_scale, "copies": copies}
        kept = lambda of: [x.detach() if isinstance(x, _Tensor) else x for x in of]
        self.grads = kept(grads)
        count = len(self.grads)
        self.sizes = []
        for name, of in kinds.items():
            of = [None] * count if of is None else kept(of)
            if len(of) != count:
                raise ValueError(f"{name}: {len(of)} tensors, expected {count}")
            setattr(self, name, of)
        self.whole = params is not None
        if self.whole and (m is None or v is None):
            raise ValueError("a step needs m and v")
        self.device = None
        self.array, self.options = (ll_tensor * max(count, 1))(), ll_adamw_options()
        self.address, self.options_address = ctypes.addressof(self.array), ctypes.addressof(self.options)
        written = set()
        for i, g in enumerate(self.grads):
            t = self.array[i]
            t.flags = self._grad_flag(g, f"grads[{i}]")
            t.n, t.grad = g.numel(), g.data_ptr()
            self.sizes.append(g.shape)
            if not self.whole:
                continue
            p = self.params[i]
            _check(p, _BF16 if isinstance(p, _Tensor) and p.dtype == _BF16 else _F32, f"params[{i}]", g.shape)
            eight = isinstance(self.m[i], _Tensor) and self.m[i].dtype == torch.float8_e4m3fn
            _check(self.m[i], torch.float8_e4m3fn if eight else _F32, f"m[{i}]", g.shape)
            _check(self.v[i], torch.float8_e5m2 if eight else _F32, f"v[{i}]", g.shape)
            blocks = (t.n + LL_STATE_BLOCK - 1) // LL_STATE_BLOCK
            for name, of in (("m_scale", self.m_scale), ("v_scale", self.v_scale)):
                if eight:
                    _check(of[i], _F32, f"{name}[{i}]", (blocks,))
                elif of[i] is not None:
                    raise ValueError(f"{name}[{i}]: states in fp32 have none")
            if self.copies[i] is not None:
                if p.dtype != _F32:
                    raise ValueError(f"copies[{i}]: only fp32 parameters have one")
                _check(self.copies[i], _BF16, f"copies[{i}]", g.shape)
            mine = [p, self.m[i], self.v[i], self.m_scale[i], self.v_scale[i], self.copies[i]]
            t.param, t.m, t.v, t.m_scale, t.v_scale, t.copy = at = [_ptr(x) for x in mine]
            t.flags |= (LL_TENSOR_PARAM_BF16 if p.dtype == _BF16 else 0) | (LL_TENSOR_STATE_8BIT if eight else 0)
            for x, a in zip(mine, at):
                if x is None:
                    continue
                if x.device != self.device:
                    raise ValueError(f"tensor {i}: on {x.device}, the first on {self.device}")
                if a and a in written:
                    raise ValueError(f"tensor {i}: the same memory is in the list twice")
                written.add(a)
        self.device = torch.device("cuda") if self.device is None else self.device

    def _grad_flag(self, g, name):
        bf16 = isinstance(g, _Tensor) and g.dtype == _BF16
        _check(g, _BF16 if bf16 else _F32, name)
        if self.device is None:
            self.device = g.device
        elif g.device != self.device:
            raise ValueError(f"{name}: on {g.device}, the first on {self.device}")
        return LL_TENSOR_GRAD_BF16 if bf16 else 0

    def set_grads(self, grads):
        """Other gradients of the same shapes (a backward pass that made new tensors).  None in a gradient's place lets its memory go: the list is then
        refused by the calls until there is another."""
        grads = list(grads)
        if len(grads) != len(self.grads):
            raise ValueError(f"grads: {len(grads)} tensors, expected {len(self.grads)}")
        if all(g is None for g in grads):
            self.grads = grads
            for t in self.array:
                t.grad = None
            return
        grads = [g.detach() if isinstance(g, _Tensor) else g for g in grads]
        flags = []
        for i, (g, size) in enumerate(zip(grads, self.sizes)):
            flags.append(0 if g is None else self._grad_flag(g, f"grads[{i}]"))
            if g is not None and g.shape != size:
                raise ValueError(f"grads[{i}]: shape {tuple(g.shape)}, expected {tuple(size)}")
        for t, g, flag in zip(self.array, grads, flags):        # (all of them or none)
            t.grad, t.flags = _ptr(g), (t.flags & ~LL_TENSOR_GRAD_BF16) | flag
        self.grads = grads

    def __len__(self):
        return len(self.grads)


def ll_grad_norm_workspace_bytes(tensors) -> int:
    return int(lib().ll_grad_norm_workspace_bytes(len(tensors)))


def ll_grad_norm(tensors, *, workspace=None, stream=None, out=None):
    """Norm of all gradients of a TensorList (or of a sequence of fp32 and bf16 tensors): [1] fp32, on the GPU."""
    if not isinstance(tensors, TensorList):
        tensors = TensorList(tensors)
    _here(tensors.device, stream, workspace, out)
    ws = _workspace(workspace, lambda: ll_grad_norm_workspace_bytes(tensors), tensors.device, stream)
    if out is None:
        out = _empty((1,), _F32, tensors.device, stream)
    else:
        _check(out, _F32, "out", (1,))
    rc = (_lib or lib()).ll_grad_norm(tensors.address, len(tensors.grads), ws.data_ptr(), ws.numel() * ws.element_size(), out.data_ptr(), _stream(stream))
    if rc != LL_OK:
        raise LLError(rc, "ll_grad_norm")
    return out


def ll_adamw(tensors, step=None, *, rate=1e-3, betas=(0.9, 0.999), eps=1e-8, decay=0.0, norm=None, max_norm=float("inf"), seed=0, clock=None,
             device_rate=None, stream=None):
    """One AdamW step over a TensorList, in place.  step: of this call, from 1; or clock: int64 [4] on the GPU, zeros to begin with, which counts
    the steps (a captured call's replays).  norm [1] fp32 (of ll_grad_norm): clipped to max_norm, and no step where it is not finite.  seed: of the
    stochastic rounding of 8-bit states and bf16 parameters.  device_rate [1] fp32: in place of rate, with a clock."""
    if not isinstance(tensors, TensorList) or not tensors.whole:
        raise TypeError("tensors: need a TensorList with params, m and v")
    if (step is None) == (clock is None):
        raise ValueError("need a step or a clock")
    if norm is not None:
        _check(norm, _F32, "norm", (1,))
    if clock is not None:
        _check(clock, torch.int64, "clock", (4,))
    if device_rate is not None:
        _check(device_rate, _F32, "device_rate", (1,))
    _here(tensors.device, stream, norm, clock, device_rate)
    o = tensors.options
    o.rate, (o.beta1, o.beta2), o.eps, o.decay, o.max_norm, o.step, o.seed = rate, betas, eps, decay, max_norm, step or 0, seed & 0xFFFFFFFF
    rc = (_lib or lib()).ll_adamw(tensors.address, len(tensors.grads), tensors.options_address, None if norm is None else norm.data_ptr(),
                                  None if clock is None else clock.data_ptr(), None if device_rate is None else device_rate.data_ptr(), _stream(stream))
    if rc != LL_OK:
        raise LLError(rc, "ll_adamw")
