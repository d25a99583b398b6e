"""Fine-tuning a fitted model on preferences or rewards (include/nmd.h).

Row i of the model L = W H scores the n columns, and softmax(L_i) is its
distribution over them.  The functions below take the scores of T rows
("logits", T x V) with one target column per row; a target below zero leaves
its row out.  They return plain CUDA tensors, the gradient of the logits
among them (there is no autograd graph: d W = grad @ H^T, d H = W^T @ grad is
the caller's).  Every call enqueues its work on torch's current stream of the
tensors' device and does not wait.  What is wrong with the arguments raises
``nmd.NmdError``.
"""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple, Optional, Sequence

import torch

from . import nmd

_DTYPES = {torch.float32: nmd.NMD_DT_FP32, torch.bfloat16: nmd.NMD_DT_BF16, torch.float16: nmd.NMD_DT_FP16}


class PreferenceLoss(NamedTuple):
    loss: torch.Tensor               # scalar
    logps: torch.Tensor              # T
    ratios: torch.Tensor             # 2 P: log ratio of each sequence to the reference
    margins: torch.Tensor            # P
    grad: Optional[torch.Tensor]     # T x V, the logits' type


class PolicyLoss(NamedTuple):
    loss: torch.Tensor               # scalar
    logps: torch.Tensor              # T
    kl: torch.Tensor                 # scalar: mean estimate of the KL divergence from the reference
    clipped: torch.Tensor            # scalar: share of the loss's weight on rows that were cut off
    grad: Optional[torch.Tensor]     # T x V, the logits' type


def _invalid(what: str):
    raise nmd.NmdError(nmd.NMD_ERR_INVALID, what)


def _matrix(x, name: str) -> int:
    """The nmd_dtype of a CUDA matrix whose rows are contiguous."""
    if not isinstance(x, torch.Tensor) or x.dim() != 2 or not x.is_cuda:
        _invalid("%s: a two-dimensional CUDA tensor is wanted" % name)
    dt = _DTYPES.get(x.dtype)
    if dt is None:
        _invalid("%s: float32, bfloat16 or float16 is wanted, not %s" % (name, x.dtype))
    if x.shape[1] < 1 or (x.shape[1] > 1 and x.stride(1) != 1):
        _invalid("%s: at least one column, and the columns of a row adjacent (stride 1)" % name)
    return dt


def _vector(v, name: str, length: int, dtype, device) -> torch.Tensor:
    if not isinstance(v, torch.Tensor) or v.dim() != 1 or v.shape[0] != length or v.dtype != dtype \
            or v.device != device:
        _invalid("%s: a %s vector of %d on %s is wanted" % (name, str(dtype).replace("torch.", ""), length, device))
    return v if v.is_contiguous() else v.contiguous()


def _offsets(offsets, device, name: str = "offsets") -> torch.Tensor:
    if not isinstance(offsets, torch.Tensor) or offsets.dim() != 1:
        _invalid("%s: a vector of sequence borders is wanted" % name)
    return _vector(offsets, name, offsets.shape[0], torch.int64, device)


def _grad_like(logits) -> torch.Tensor:
    """The gradient's tensor: the logits' row stride, so that both are reached by the same 16-byte vectors."""
    T, V = logits.shape
    ld = logits.stride(0) if T > 1 else V
    if ld <= V:
        return torch.empty((T, V), dtype=logits.dtype, device=logits.device)
    return torch.empty((T, ld), dtype=logits.dtype, device=logits.device)[:, :V]


def _stream(device) -> int:
    return torch.cuda.current_stream(device).cuda_stream


def _call(device, name: str, *args):
    with torch.cuda.device(device):
        st = getattr(nmd.lib(), name)(*args, _stream(device))
    if st != nmd.NMD_OK:
        nmd._check(None, st, name)


def _bytes(name: str, *args) -> int:
    out = C.c_size_t(0)
    nmd._check(None, getattr(nmd.lib(), name)(*args, C.byref(out)), name)
    return out.value


def token_logprobs(logits, targets, *, temperature: float = 1.0) -> torch.Tensor:
    """log softmax(logits / temperature) at one column per row (T fp32; 0 where the target is below zero)."""
    dt = _matrix(logits, "logits")
    T, V = logits.shape
    targets = _vector(targets, "targets", T, torch.int64, logits.device)
    logps = torch.empty(T, dtype=torch.float32, device=logits.device)
    _call(logits.device, "nmd_token_logprobs", logits.data_ptr(), dt, T, V, logits.stride(0), targets.data_ptr(),
          temperature, logps.data_ptr())
    return logps


def factor_logprobs(A, B, targets, *, temperature: float = 1.0) -> torch.Tensor:
    """token_logprobs of the scores A @ B^T without forming them (T fp32).

    ``A`` (T x r) and ``B`` (n x r, r <= 256) have one type and any strides: the model's rows are A = W[rows] and
    B = H.t().  16-bit factors are read where they are if their rows are contiguous, 16-byte aligned and a multiple
    of 8 elements apart; others are packed first.
    """
    for x, name in ((A, "A"), (B, "B")):
        if not isinstance(x, torch.Tensor) or x.dim() != 2 or not x.is_cuda or x.dtype not in _DTYPES:
            _invalid("%s: a two-dimensional float32, bfloat16 or float16 CUDA tensor is wanted" % name)
    device, (T, r), n = A.device, A.shape, B.shape[0]
    if B.device != device or B.dtype != A.dtype or B.shape[1] != r:
        _invalid("B: %s of %d columns on %s is wanted, as A" % (A.dtype, r, device))
    if not 1 <= r <= 256 or n < 1:
        _invalid("A, B: 1 to 256 columns and at least one row of B are wanted")
    targets = _vector(targets, "targets", T, torch.int64, device)
    logps = torch.empty(T, dtype=torch.float32, device=device)
    factors = (A.data_ptr(), *A.stride(), B.data_ptr(), *B.stride(), _DTYPES[A.dtype], T, n, r)
    nbytes = _bytes("nmd_factor_workspace_bytes", *factors)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    _call(device, "nmd_factor_logprobs", *factors, targets.data_ptr(), temperature, logps.data_ptr(), ws.data_ptr(),
          nbytes)
    return logps


def preference_loss(logits, targets, offsets, reference, *, beta: float = 0.1, label_smoothing: float = 0.0,
                    average: bool = False, temperature: float = 1.0, grad: bool = True) -> PreferenceLoss:
    """Paired preference loss -log sigma(beta (R_chosen - R_rejected)), mean over the pairs, and its gradient.

    The sequences are packed into the rows of ``logits``: sequence k is rows ``offsets[k]`` to ``offsets[k + 1]``
    (int64, 2 P + 1 ascending borders), and pair p prefers sequence 2 p to sequence 2 p + 1.  R is the sum (or, with
    ``average``, the mean) over a sequence's live rows of the log-probability less ``reference``, the reference
    model's log-probability of the same column (fp32, one per row).
    """
    dt = _matrix(logits, "logits")
    device, (T, V) = logits.device, logits.shape
    targets = _vector(targets, "targets", T, torch.int64, device)
    reference = _vector(reference, "reference", T, torch.float32, device)
    offsets = _offsets(offsets, device)
    P = offsets.shape[0] // 2
    if offsets.shape[0] != 2 * P + 1 or P < 1:
        _invalid("offsets: 2 P + 1 borders of P >= 1 pairs are wanted, got %d" % offsets.shape[0])
    nbytes = _bytes("nmd_preference_workspace_bytes", T, P)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    out = torch.empty(1 + T + 3 * P, dtype=torch.float32, device=device)
    loss, logps, ratios, margins = out[0], out[1:1 + T], out[1 + T:1 + T + 2 * P], out[1 + T + 2 * P:]
    g = _grad_like(logits) if grad else None
    _call(device, "nmd_preference_loss", logits.data_ptr(), dt, T, V, logits.stride(0), targets.data_ptr(),
          offsets.data_ptr(), P, reference.data_ptr(), beta, label_smoothing, int(average), temperature,
          loss.data_ptr(), logps.data_ptr(), ratios.data_ptr(), margins.data_ptr(), g.data_ptr() if grad else None,
          g.stride(0) if grad else 0, ws.data_ptr(), nbytes)
    return PreferenceLoss(loss, logps, ratios, margins, g)


def policy_loss(logits, targets, old, reference, advantages, *, offsets=None, clip_low: float = 0.2,
                clip_high: float = 0.2, kl_coef: float = 0.0, temperature: float = 1.0,
                grad: bool = True) -> PolicyLoss:
    """Clipped policy loss with a KL term, and its gradient.

    ``old``, ``reference`` and ``advantages`` hold one fp32 value per row: the column's log-probability under the
    policy that produced it and under the reference model (None where ``kl_coef`` is 0), and its advantage.  Without
    ``offsets`` the loss is the mean over the live rows; with the borders of sequences (int64, S + 1 ascending) it is
    the mean over the sequences of each one's mean.
    """
    dt = _matrix(logits, "logits")
    device, (T, V) = logits.device, logits.shape
    targets = _vector(targets, "targets", T, torch.int64, device)
    old = _vector(old, "old", T, torch.float32, device)
    advantages = _vector(advantages, "advantages", T, torch.float32, device)
    if reference is not None:
        reference = _vector(reference, "reference", T, torch.float32, device)
    elif kl_coef != 0:
        _invalid("reference: wanted with a KL term")
    S = 0
    if offsets is not None:
        offsets = _offsets(offsets, device)
        S = offsets.shape[0] - 1
        if S < 1:
            _invalid("offsets: S + 1 borders of S >= 1 sequences are wanted")
    nbytes = _bytes("nmd_policy_workspace_bytes", T)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    out = torch.empty(3 + T, dtype=torch.float32, device=device)
    g = _grad_like(logits) if grad else None
    _call(device, "nmd_policy_loss", logits.data_ptr(), dt, T, V, logits.stride(0), targets.data_ptr(),
          old.data_ptr(), None if reference is None else reference.data_ptr(), advantages.data_ptr(),
          None if offsets is None else offsets.data_ptr(), S, clip_low, clip_high, kl_coef, temperature,
          out.data_ptr(), out[3:].data_ptr() if T else None, g.data_ptr() if grad else None,
          g.stride(0) if grad else 0, ws.data_ptr(), nbytes)
    return PolicyLoss(out[0], out[3:], out[1], out[2], g)


def _dense(x) -> bool:
    """Whether the elements fill one span of memory in some order of the dimensions."""
    if x.is_contiguous():
        return True
    want = 1
    for stride, size in sorted((s, n) for s, n in zip(x.stride(), x.shape) if n > 1):
        if stride != want:
            return False
        want *= size
    return True


def clip_grad_norm(grads: Sequence[torch.Tensor], max_norm: float,
                   out: Optional[Sequence[torch.Tensor]] = None) -> torch.Tensor:
    """Global 2-norm of ``grads`` (a scalar tensor), and the gradients scaled by min(1, max_norm / norm): in place, or
    into ``out`` (tensors of the gradients' types, shapes and strides).  CUDA tensors of one device without gaps
    (contiguous, or contiguous after a permutation of the dimensions)."""
    grads = list(grads)
    if not grads or not isinstance(grads[0], torch.Tensor):
        _invalid("grads: at least one tensor is wanted")
    device, count = grads[0].device, len(grads)
    outs = grads if out is None else list(out)
    if len(outs) != count:
        _invalid("out: %d tensors are wanted, got %d" % (count, len(outs)))
    ptrs, sizes = (C.c_void_p * count)(), (C.c_int64 * count)()
    optrs, kinds = (C.c_void_p * count)(), (C.c_int32 * count)()
    for k, (x, o) in enumerate(zip(grads, outs)):
        dt = _DTYPES.get(x.dtype)
        if dt is None or not x.is_cuda or x.device != device or not _dense(x):
            _invalid("grads[%d]: a float32, bfloat16 or float16 tensor without gaps on %s is wanted" % (k, device))
        if o is not x and (o.dtype != x.dtype or o.device != device or o.shape != x.shape
                           or o.stride() != x.stride()):
            _invalid("out[%d]: a tensor of its gradient's type, shape, strides and device is wanted" % k)
        ptrs[k], optrs[k], sizes[k], kinds[k] = x.data_ptr(), o.data_ptr(), x.numel(), dt
    norm = torch.empty((), dtype=torch.float32, device=device)
    nbytes = _bytes("nmd_clip_workspace_bytes", count)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    _call(device, "nmd_clip_grad_norm", count, ptrs, sizes, kinds, max_norm, None if out is None else optrs,
          norm.data_ptr(), ws.data_ptr(), nbytes)
    return norm
