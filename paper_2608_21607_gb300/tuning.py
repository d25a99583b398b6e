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

import array
import ctypes as C
import functools
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
    V = x.shape[1]
    if V < 1 or (V > 1 and x.stride(1) != 1):
        _invalid("%s: at least one column, and the columns of a row adjacent (stride 1)" % name)
    return dt


def _vector(v, name: str, length: int, dtype, index: int) -> torch.Tensor:
    if not isinstance(v, torch.Tensor) or v.dim() != 1 or v.numel() != length or v.dtype != dtype \
            or not v.is_cuda or v.get_device() != index:
        _invalid("%s: a %s vector of %d on cuda:%d is wanted" % (name, str(dtype).replace("torch.", ""), length, index))
    return v if v.is_contiguous() else v.contiguous()


def _offsets(offsets, index: int, name: str = "offsets") -> torch.Tensor:
    if not isinstance(offsets, torch.Tensor) or offsets.dim() != 1:
        _invalid("%s: a vector of sequence borders is wanted" % name)
    return _vector(offsets, name, offsets.numel(), torch.int64, index)


def _grad_like(logits, T: int, V: int, ld: int) -> torch.Tensor:
    """The gradient's tensor: rows whose distance differs from the logits' by whole 128-byte lines, so that both are
    reached by the same vectors and padded rows are written in whole lines; less than a line of padding, however far
    apart the logits' rows lie.  (By whole 16-byte vectors only, 4096 rows of 139,255 of 139,264 bf16 columns take
    398.5 us instead of 396.5.)"""
    pad = (ld - V) % (128 // logits.element_size()) if T > 1 and ld > V else 0
    if pad == 0:
        return torch.empty((T, V), dtype=logits.dtype, device=logits.device)
    return torch.empty((T, V + pad), dtype=logits.dtype, device=logits.device)[:, :V]


_calls = {}


def _call(index: int, name: str, *args):
    """The C call of that name with the stream that is current on the device, and its status checked."""
    f = _calls.get(name)
    if f is None:
        f = _calls[name] = getattr(nmd.lib(), name)
    if torch._C._cuda_getDevice() == index:
        st = f(*args, torch._C._cuda_getCurrentRawStream(index))
    else:
        with torch.cuda.device(index):
            st = f(*args, torch._C._cuda_getCurrentRawStream(index))
    if st != nmd.NMD_OK:
        nmd._check(None, st, name)


@functools.lru_cache(maxsize=256)
def _bytes_of_sizes(name: str, *sizes) -> int:
    out = C.c_size_t(0)
    nmd._check(None, getattr(nmd.lib(), name)(*sizes, C.byref(out)), name)
    return out.value


def token_logprobs(logits, targets, *, temperature: float = 1.0) -> torch.Tensor:
    """log softmax(logits / temperature) at one column per row (T fp32; 0 where the target is below zero)."""
    dt = _matrix(logits, "logits")
    index, (T, V) = logits.get_device(), logits.shape
    targets = _vector(targets, "targets", T, torch.int64, index)
    logps = torch.empty(T, dtype=torch.float32, device=logits.device)
    _call(index, "nmd_token_logprobs", logits.data_ptr(), dt, T, V, logits.stride(0), targets.data_ptr(), temperature,
          logps.data_ptr())
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
    device, index, (T, r), n = A.device, A.get_device(), A.shape, B.shape[0]
    if B.device != device or B.dtype != A.dtype or B.shape[1] != r:
        _invalid("B: %s of %d columns on %s is wanted, as A" % (A.dtype, r, device))
    if not 1 <= r <= 256 or n < 1:
        _invalid("A, B: 1 to 256 columns and at least one row of B are wanted")
    targets = _vector(targets, "targets", T, torch.int64, index)
    logps = torch.empty(T, dtype=torch.float32, device=device)
    a, b, shape = A.data_ptr(), B.data_ptr(), (*B.stride(), _DTYPES[A.dtype], T, n, r)
    # the size goes by the sizes, strides and alignments alone
    nbytes = _bytes_of_sizes("nmd_factor_workspace_bytes", a & 15, *A.stride(), b & 15, *shape)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    _call(index, "nmd_factor_logprobs", a, *A.stride(), b, *shape, targets.data_ptr(), temperature, logps.data_ptr(), ws.data_ptr(),
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
    device, index, (T, V), ld = logits.device, logits.get_device(), logits.shape, logits.stride(0)
    targets = _vector(targets, "targets", T, torch.int64, index)
    reference = _vector(reference, "reference", T, torch.float32, index)
    offsets = _offsets(offsets, index)
    P = offsets.numel() // 2
    if offsets.numel() != 2 * P + 1 or P < 1:
        _invalid("offsets: 2 P + 1 borders of P >= 1 pairs are wanted, got %d" % offsets.numel())
    nbytes = _bytes_of_sizes("nmd_preference_workspace_bytes", T, P)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    loss = torch.empty((), dtype=torch.float32, device=device)   # its own: a loss that is kept keeps nothing else
    logps = torch.empty(T, dtype=torch.float32, device=device)
    ratios = torch.empty(2 * P, dtype=torch.float32, device=device)
    margins = torch.empty(P, dtype=torch.float32, device=device)
    g = _grad_like(logits, T, V, ld) if grad else None
    _call(index, "nmd_preference_loss", logits.data_ptr(), dt, T, V, ld, targets.data_ptr(), offsets.data_ptr(), P,
          reference.data_ptr(), beta, label_smoothing, int(average), temperature, loss.data_ptr(), logps.data_ptr(),
          ratios.data_ptr(), margins.data_ptr(), g.data_ptr() if grad else None, g.stride(0) if grad else 0,
          ws.data_ptr(), nbytes)
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
    device, index, (T, V), ld = logits.device, logits.get_device(), logits.shape, logits.stride(0)
    targets = _vector(targets, "targets", T, torch.int64, index)
    old = _vector(old, "old", T, torch.float32, index)
    advantages = _vector(advantages, "advantages", T, torch.float32, index)
    if reference is not None:
        reference = _vector(reference, "reference", T, torch.float32, index)
    elif kl_coef != 0:
        _invalid("reference: wanted with a KL term")
    S = 0
    if offsets is not None:
        offsets = _offsets(offsets, index)
        S = offsets.numel() - 1
        if S < 1:
            _invalid("offsets: S + 1 borders of S >= 1 sequences are wanted")
    nbytes = _bytes_of_sizes("nmd_policy_workspace_bytes", T)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    stats = torch.empty(3, dtype=torch.float32, device=device)   # their own: results that are kept keep nothing else
    logps = torch.empty(T, dtype=torch.float32, device=device)
    g = _grad_like(logits, T, V, ld) if grad else None
    _call(index, "nmd_policy_loss", logits.data_ptr(), dt, T, V, ld, targets.data_ptr(), old.data_ptr(),
          None if reference is None else reference.data_ptr(), advantages.data_ptr(),
          None if offsets is None else offsets.data_ptr(), S, clip_low, clip_high, kl_coef, temperature,
          stats.data_ptr(), logps.data_ptr(), g.data_ptr() if grad else None, g.stride(0) if grad else 0,
          ws.data_ptr(), nbytes)
    return PolicyLoss(stats[0], logps, stats[1], stats[2], g)


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
    into ``out`` (tensors of the gradients' types and sizes).  CUDA tensors of one device without gaps
    (contiguous, or contiguous after a permutation of the dimensions); one that is written overlaps no other."""
    grads = list(grads)
    outs = grads if out is None else list(out)
    count, Tensor = len(grads), torch.Tensor
    if count == 0 or len(outs) != count:
        _invalid("grads, out: as many tensors as gradients are wanted, and at least one")
    try:   # (maps over methods: a list of hundreds of tensors costs about half a microsecond each)
        devices = set(map(Tensor.get_device, grads)) | set(map(Tensor.get_device, outs))
        sizes = array.array("q", map(Tensor.numel, grads))
        adjacent = all(map(Tensor.is_contiguous, grads)) and all(map(Tensor.is_contiguous, outs))
    except TypeError:
        _invalid("grads, out: tensors are wanted")
    device = grads[0].device
    if device.type != "cuda" or len(devices) != 1:
        _invalid("grads, out: tensors of one CUDA device are wanted")
    types = [x.dtype for x in grads]
    if not _DTYPES.keys() >= set(types) or not (adjacent or all(map(_dense, grads))):
        _invalid("grads: float32, bfloat16 or float16 tensors without gaps are wanted")
    if outs is not grads and (types != [x.dtype for x in outs] or sizes != array.array("q", map(Tensor.numel, outs))
                              or not (adjacent or all(x.shape == o.shape and x.stride() == o.stride()
                                                      for x, o in zip(grads, outs)))):
        _invalid("out: each tensor has its gradient's type and, unless all are contiguous, its shape and strides")
    kinds = array.array("i", [_DTYPES[t] for t in types])
    ptrs = array.array("Q", map(Tensor.data_ptr, grads))
    optrs = None if out is None else array.array("Q", map(Tensor.data_ptr, outs))
    norm = torch.empty((), dtype=torch.float32, device=device)
    nbytes = _bytes_of_sizes("nmd_clip_workspace_bytes", count)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    _call(norm.get_device(), "nmd_clip_grad_norm", count, ptrs.buffer_info()[0], sizes.buffer_info()[0],
          kinds.buffer_info()[0], max_norm, None if out is None else optrs.buffer_info()[0], norm.data_ptr(),
          ws.data_ptr(), nbytes)
    torch.autograd.graph.increment_version(outs)   # autograd has to know that a tensor it may have saved has changed
    return norm
