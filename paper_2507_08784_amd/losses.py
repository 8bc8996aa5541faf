"""Losses over a language model's logits, and their gradients, on MI355X
(include/greedylore_losses.h): what makes the gradients that the compression
step takes.

    from paper_2507_08784_amd import losses

    r = losses.token_logprobs(logits, targets)                    # r.logps
    r = losses.preference_loss(logits, targets, ref, beta=0.1)    # r.loss.backward()
    r = losses.policy_loss(logits, targets, old, advantages, ref_logps=ref, kl_coef=0.04)
    r = losses.distill_loss(logits, teacher_ids, teacher_logits, temperature=2.0)

`logits` are (rows, V) or (batch, steps, V), fp32, bf16 or fp16, with any
strides as long as a row is contiguous: `model(ids)[:, :-1]` against
`labels[:, 1:]` is taken as it is.  `targets` (int32 or int64) have the
logits' shape without V; a row whose target is `ignore_index` is not trained
on: nothing of it is read, and its gradient is zero.  Arrays beside the
targets (fp32) have their shape and may be expanded (`adv[:, None].expand(B, S)`).

The gradient with respect to the logits comes in one of two ways:

  autograd   if the logits require a gradient, `loss` (or `logps`) is part of
             the graph; the losses compute the gradient in the forward call
             (one pass over the logits gives both) and backward hands it on,
             times the upstream gradient (a factor other than a power of two
             rounds bf16 and fp16 gradients a second time: pass it as
             `grad_scale` instead, with which the gradient is made)
  explicit   grad=True (weights=... of token_logprobs) returns it as `dlogits`;
             nothing is recorded

`out` is a tensor for the gradient, of the logits' shape and type; it may be
the logits themselves, which the gradient then replaces.  All work is enqueued
on the current stream of the logits' device; nothing waits for the GPU.
Workspaces and results come from torch's allocator.  There is no CPU path.
"""
from __future__ import annotations

import ctypes
import struct
from collections import namedtuple

import torch

from . import _check, load

LOSS_EXPORTED = (
    "glr_loss_workspace_bytes", "glr_token_logprobs", "glr_token_logprobs_backward",
    "glr_preference_loss", "glr_policy_loss", "glr_distill_loss", "glr_loss_rescale",
)
KINDS = {"sigmoid": 0, "hinge": 1, "squared": 2}
REDUCTIONS = {"token": 0, "sequence": 1}
_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_ITYPES = {torch.int32: 0, torch.int64: 1}
_PREFERENCE, _POLICY, _DISTILL = 1, 2, 3

TokenLogprobs = namedtuple("TokenLogprobs", "logps dlogits")
PreferenceLoss = namedtuple("PreferenceLoss", "loss logps rewards dlogits")
PolicyLoss = namedtuple("PolicyLoss", "loss logps kl clipped dlogits")
DistillLoss = namedtuple("DistillLoss", "loss losses dlogits")

_I32, _I64, _F64, _VP = ctypes.c_int32, ctypes.c_int64, ctypes.c_double, ctypes.c_void_p


class RowArray(ctypes.Structure):
    _fields_ = [("data", _VP), ("stride_b", _I64), ("stride_s", _I64)]


class Rows(ctypes.Structure):
    _fields_ = [
        ("batch", _I64), ("steps", _I64), ("vocab", _I64), ("logits", RowArray), ("dlogits", RowArray),
        ("dtype", _I32), ("target_type", _I32), ("targets", RowArray), ("ignore_index", _I64),
        ("temperature", _F64), ("grad_scale", _F64),
    ]


class Seqs(ctypes.Structure):
    _fields_ = [("seqs", _I64), ("cu_seqlens", _VP), ("cu_type", _I32)]


class PrefArgs(ctypes.Structure):
    _fields_ = [("seqs", Seqs), ("kind", _I32), ("average", _I32), ("beta", _F64), ("label_smoothing", _F64),
                ("ref_logps", _VP), ("loss", _VP), ("logps", _VP), ("rewards", _VP)]


class PolicyArgs(ctypes.Structure):
    _fields_ = [("seqs", Seqs), ("reduction", _I32), ("clip_low", _F64), ("clip_high", _F64), ("kl_coef", _F64),
                ("denominator", _F64), ("old_logps", RowArray), ("advantages", RowArray), ("ref_logps", RowArray),
                ("loss", _VP), ("kl", _VP), ("clipped", _VP), ("logps", _VP)]


class DistillArgs(ctypes.Structure):
    _fields_ = [("top", _I32), ("id_type", _I32), ("teacher_type", _I32), ("ids", RowArray), ("teacher", RowArray),
                ("teacher_lse", RowArray), ("hard_weight", _F64), ("denominator", _F64), ("loss", _VP),
                ("losses", _VP)]


# The same structs as packed bytes: what a call passes (a nested ctypes struct
# takes several microseconds to fill, about what a small launch takes).
_ROWS = struct.Struct("@3qPqqPqqiiPqqqdd").pack
_PREF = struct.Struct("@qPi4xiidd4P").pack
_POLICY_ARGS = struct.Struct("@qPi4xi4x4dPqqPqqPqq4P").pack
_DISTILL_ARGS = struct.Struct("@iii4xPqqPqqPqqdd2P").pack
_ARRAY = struct.Struct("@Pqq").pack

_fns = None
_fast = {}
_sizes = {}


def _lib():
    """The library with the losses' prototypes (structs by reference)."""
    global _fns
    if _fns is None:
        lib = load()
        P, S = ctypes.POINTER, ctypes.c_size_t
        sig = {
            "glr_loss_workspace_bytes": [P(Rows), _I32, _I64, P(S)],
            "glr_token_logprobs": [P(Rows), P(RowArray), _VP, _VP, _VP, S, _VP],
            "glr_token_logprobs_backward": [P(Rows), _VP, P(RowArray), _VP],
            "glr_preference_loss": [P(Rows), P(PrefArgs), _VP, S, _VP],
            "glr_policy_loss": [P(Rows), P(PolicyArgs), _VP, S, _VP],
            "glr_distill_loss": [P(Rows), P(DistillArgs), _VP, S, _VP],
            "glr_loss_rescale": [_VP, _I64, _I32, _VP, _VP],
        }
        for name, args in sig.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = _I32, args
            # and one that takes the packed structs
            fast = lib[name]
            fast.restype = _I32
            fast.argtypes = [ctypes.c_char_p if a in (P(Rows), P(RowArray), P(PrefArgs), P(PolicyArgs), P(DistillArgs))
                             else a for a in args]
            _fast[name] = fast
        _fns = lib
    return _fns


def _run(name, device, *args):
    """Calls an entry on the device's current stream."""
    if _fns is None:
        _lib()
    index = device.index
    if index == torch._C._cuda_getDevice():
        status = _fast[name](*args, torch._C._cuda_getCurrentRawStream(index))
    else:
        with torch.cuda.device(device):
            status = _fast[name](*args, torch._C._cuda_getCurrentRawStream(index))
    if status:
        _check(status)


def _workspace(op, rows, count, seqs, grad, device):
    """Scratch of a call and its size."""
    key = (op, count, seqs, grad)
    size = _sizes.get(key)
    if size is None:
        if _fns is None:
            _lib()
        n = ctypes.c_size_t()
        _check(_fast["glr_loss_workspace_bytes"](rows, op, seqs, n))
        if len(_sizes) > 4096:
            _sizes.clear()
        size = _sizes[key] = n.value
    return torch.empty(size, dtype=torch.uint8, device=device), size


# ----------------------------------------------------------------------------
# arguments
# ----------------------------------------------------------------------------
_NONE = (0, 0, 0)
_FLOAT = (torch.float32,)
_INT = (torch.int64, torch.int32)
_ANY = (torch.float32, torch.bfloat16, torch.float16)


def _same(x, name, shape, device, dtypes):
    if not isinstance(x, torch.Tensor):
        raise TypeError(f"{name} must be a tensor, not {type(x).__name__}")
    if x.dtype not in dtypes:
        raise TypeError(f"{name} must be {' or '.join(str(d) for d in dtypes)}, not {x.dtype}")
    if x.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, not {tuple(x.shape)}")
    if x.device != device:
        raise ValueError(f"{name} must live on {device}, not {x.device}")


def _array(x, name, shape, device, dtypes=_FLOAT):
    """(pointer, batch stride, step stride) of an array over the rows."""
    _same(x, name, shape, device, dtypes)
    st = x.stride()
    return (x.data_ptr(), st[0], st[1]) if len(st) == 2 else (x.data_ptr(), 0, st[0])


def _lists(x, name, shape, device, dtypes):
    """The same of an array with a contiguous list in each row."""
    _same(x, name, shape, device, dtypes)
    st = x.stride()
    if st[-1] != 1 and shape[-1] > 1:
        raise ValueError(f"a row of {name} must be contiguous" + (" (stride 1 over the vocabulary)" if dtypes is _ANY else ""))
    return (x.data_ptr(), st[0], st[1]) if len(st) == 3 else (x.data_ptr(), 0, st[0])


def _rows(logits, targets, ignore_index, temperature, grad, grad_scale, out):
    """The checks that every loss makes of its rows: (packed struct, shape of
    the rows, device, (batch, steps), gradient or None)."""
    if not isinstance(logits, torch.Tensor):
        raise TypeError(f"logits must be a tensor, not {type(logits).__name__}")
    dtype = logits.dtype
    if dtype not in _DTYPES:
        raise TypeError(f"logits must be float32, bfloat16 or float16, not {dtype}")
    full = logits.shape
    if len(full) not in (2, 3):
        raise ValueError(f"logits must be (rows, vocab) or (batch, steps, vocab), not {tuple(full)}")
    if not logits.is_cuda:
        raise ValueError("the losses run on the GPU only (logits on the CPU)")
    shape, device = full[:-1], logits.device
    z = _lists(logits, "logits", full, device, _ANY)
    d, dz = None, _NONE
    if grad:
        if out is None:
            d = torch.empty(full, dtype=dtype, device=device)
        else:
            _same(out, "out", full, device, (dtype,))
            if out.data_ptr() == z[0] and out.stride() != logits.stride():
                raise ValueError("out that replaces the logits must have their strides")
            d = out
        dz = _lists(d, "out", full, device, _ANY)
    elif out is not None:
        raise ValueError("out is the gradient's: it needs grad=True (weights=... of token_logprobs)")
    y, itype = _NONE, 0
    if targets is not None:
        y = _array(targets, "targets", shape, device, _INT)
        itype = _ITYPES[targets.dtype]
    b, s = shape if len(shape) == 2 else (1, shape[0])
    return (_ROWS(b, s, full[-1], *z, *dz, _DTYPES[dtype], itype, *y, ignore_index, temperature, grad_scale), shape,
            device, (b, s), d)


def _seqs(cu, shape, device):
    """(sequences, pointer of their offsets, type of them)."""
    if cu is None:
        if len(shape) != 2:
            raise ValueError("packed rows (2-D logits) need cu_seqlens")
        return shape[0], 0, 0
    if cu.dim() != 1 or cu.numel() < 2:
        raise ValueError("cu_seqlens must be one-dimensional with at least two offsets")
    if len(shape) != 1:
        raise ValueError("cu_seqlens goes with packed rows (2-D logits)")
    _same(cu, "cu_seqlens", cu.shape, device, _INT)
    if not cu.is_contiguous():
        raise ValueError("cu_seqlens must be contiguous")
    return cu.numel() - 1, cu.data_ptr(), _ITYPES[cu.dtype]


def _records(logits, grad):
    """Whether a call is part of the graph (and not an explicit one)."""
    return not grad and isinstance(logits, torch.Tensor) and logits.requires_grad and torch.is_grad_enabled()


# ----------------------------------------------------------------------------
# autograd
# ----------------------------------------------------------------------------
class _WithGradient(torch.autograd.Function):
    """A loss whose gradient came with it; backward hands it on once, times
    the upstream gradient."""

    @staticmethod
    def forward(ctx, logits, compute):
        result = compute()
        ctx.dlogits = result.dlogits
        rest = tuple(result[1:-1])
        ctx.mark_non_differentiable(*rest)
        return (result.loss,) + rest

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_loss, *_):
        d, ctx.dlogits = ctx.dlogits, None
        if d is None:
            raise RuntimeError("the loss's gradient was handed on already: call the loss again for a second backward")
        scale = grad_loss.float().contiguous()
        if d.is_contiguous():
            _run("glr_loss_rescale", d.device, d.data_ptr(), d.numel(), _DTYPES[d.dtype], scale.data_ptr())
        else:                       # an `out` with room between its rows
            d.mul_(scale)
        return d, None


class _TokenLogprobs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, targets, temperature, ignore_index):
        rows, shape, device, (b, s), _ = _rows(logits, targets, ignore_index, temperature, False, 1.0, None)
        logps = torch.empty(shape, dtype=torch.float32, device=device)
        stats = torch.empty((b * s, 2), dtype=torch.float32, device=device)
        _run("glr_token_logprobs", device, rows, None, logps.data_ptr(), stats.data_ptr(), None, 0)
        ctx.save_for_backward(logits, targets, stats)
        ctx.options = (ignore_index, temperature)
        return logps

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad):
        logits, targets, stats = ctx.saved_tensors
        rows, shape, device, _, d = _rows(logits, targets, *ctx.options, True, 1.0, None)
        w = _ARRAY(*_array(grad, "the upstream gradient", shape, device))
        _run("glr_token_logprobs_backward", device, rows, stats.data_ptr(), w)
        return d, None, None, None


# ----------------------------------------------------------------------------
# the losses
# ----------------------------------------------------------------------------
def token_logprobs(logits, targets, *, weights=None, temperature=1.0, ignore_index=-100, grad_scale=1.0, out=None):
    """log softmax(logits / temperature) of each row's target: logps (fp32, 0
    where ignored).  With weights (fp32, of the targets' shape) also dlogits,
    grad_scale times the gradient of sum(weights * logps), from the same pass
    over the logits: weights of -1 / count are the mean cross entropy."""
    if weights is None and _records(logits, False):
        if out is not None:
            raise ValueError("out needs weights")
        return TokenLogprobs(_TokenLogprobs.apply(logits, targets, temperature, ignore_index), None)
    rows, shape, device, _, d = _rows(logits, targets, ignore_index, temperature, weights is not None, grad_scale, out)
    w = _ARRAY(*_array(weights, "weights", shape, device)) if weights is not None else None
    logps = torch.empty(shape, dtype=torch.float32, device=device)
    _run("glr_token_logprobs", device, rows, w, logps.data_ptr(), None, None, 0)
    return TokenLogprobs(logps, d)


def preference_loss(logits, targets, ref_logps, *, beta=0.1, kind="sigmoid", label_smoothing=0.0, average=False,
                    cu_seqlens=None, ignore_index=-100, grad=False, grad_scale=1.0, out=None):
    """Loss of P pairs of sequences, the chosen ones first, then the rejected
    ones in the same order: (2P, steps, V) logits, or packed rows (rows, V)
    with cu_seqlens (2P + 1 offsets).  ref_logps: 2P fp32, the reference
    model's sums (means with average=True) of the sequences' log-probabilities.
    With D the chosen minus the rejected log ratio to the reference and
    h = beta D, kind "sigmoid" is -log sigma(h) (smoothed by label_smoothing),
    "hinge" max(0, 1 - h), "squared" (D - 1 / (2 beta))^2; the mean over pairs.
    Returns loss, logps (2P), rewards = beta (logps - ref_logps), dlogits."""
    if kind not in KINDS:
        raise ValueError(f"kind must be one of {sorted(KINDS)}, not {kind!r}")
    record = _records(logits, grad)

    def compute():
        rows, shape, device, (b, s), d = _rows(logits, targets, ignore_index, 1.0, grad or record, grad_scale, out)
        n, *seqs = _seqs(cu_seqlens, shape, device)
        _same(ref_logps, "ref_logps", (n,), device, _FLOAT)
        if not ref_logps.is_contiguous():
            raise ValueError("ref_logps must be contiguous")
        logps, rewards = torch.empty((2, n), dtype=torch.float32, device=device).unbind()
        loss = torch.empty((), dtype=torch.float32, device=device)
        at = logps.data_ptr()
        args = _PREF(n, *seqs, KINDS[kind], bool(average), beta, label_smoothing, ref_logps.data_ptr(), loss.data_ptr(),
                     at, at + 4 * n)
        ws, size = _workspace(_PREFERENCE, rows, b * s, n, d is not None, device)
        _run("glr_preference_loss", device, rows, args, ws.data_ptr(), size)
        return PreferenceLoss(loss, logps, rewards, d)

    if record:
        return PreferenceLoss(*_WithGradient.apply(logits, compute), None)
    return compute()


def policy_loss(logits, targets, old_logps, advantages, *, ref_logps=None, clip_low=0.2, clip_high=0.2, kl_coef=0.0,
                reduction="token", denominator=None, cu_seqlens=None, temperature=1.0, ignore_index=-100, grad=False,
                grad_scale=1.0, out=None):
    """The clipped surrogate with a KL term: with r = exp(logp - old) and
    d = ref - logp, the mean over the rows trained on of
    -min(r A, clip(r, 1 - clip_low, 1 + clip_high) A) + kl_coef (e^d - d - 1);
    the mean over all of them (reduction "token"; `denominator`, a number,
    takes the place of their count, as a batch spread over several ranks needs) or of
    each sequence first and then over the sequences ("sequence": 3-D logits, or
    cu_seqlens).  Returns loss, logps, kl (the mean of e^d - d - 1), clipped (the share
    of rows on the clipped side), dlogits."""
    if reduction not in REDUCTIONS:
        raise ValueError(f"reduction must be one of {sorted(REDUCTIONS)}, not {reduction!r}")
    if denominator is not None and not denominator > 0:
        raise ValueError(f"denominator must be > 0, not {denominator!r}")
    record = _records(logits, grad)

    def compute():
        rows, shape, device, (b, s), d = _rows(logits, targets, ignore_index, temperature, grad or record, grad_scale, out)
        seqs = (0, 0, 0)
        if cu_seqlens is not None or reduction == "sequence":
            seqs = _seqs(cu_seqlens, shape, device)
        old, adv = _array(old_logps, "old_logps", shape, device), _array(advantages, "advantages", shape, device)
        ref = _array(ref_logps, "ref_logps", shape, device) if ref_logps is not None else _NONE
        loss, kl, clipped = torch.empty(3, dtype=torch.float32, device=device).unbind()
        logps = torch.empty(shape, dtype=torch.float32, device=device)
        at = loss.data_ptr()
        args = _POLICY_ARGS(*seqs, REDUCTIONS[reduction], clip_low, clip_high, kl_coef, denominator or 0.0, *old, *adv,
                            *ref, at, at + 4, at + 8, logps.data_ptr())
        ws, size = _workspace(_POLICY, rows, b * s, seqs[0], d is not None, device)
        _run("glr_policy_loss", device, rows, args, ws.data_ptr(), size)
        return PolicyLoss(loss, logps, kl, clipped, d)

    if record:
        return PolicyLoss(*_WithGradient.apply(logits, compute), None)
    return compute()


def distill_loss(logits, teacher_ids, teacher_logits, *, temperature=1.0, teacher_lse=None, targets=None,
                 hard_weight=0.0, denominator=None, ignore_index=-100, grad=False, grad_scale=1.0, out=None):
    """Distillation from a teacher's top logits: teacher_ids (int) and
    teacher_logits (fp32, bf16 or fp16) have the logits' shape with K entries
    in the place of V; an entry with a negative index or a logit of -inf is
    absent.  With p the teacher's softmax at `temperature` over its entries and
    q the student's over the vocabulary, a row's loss is
    (1 - hard_weight) temperature^2 sum p (log p - log q) + hard_weight times
    the cross entropy of its target.  teacher_lse (fp32, log sum exp of the
    teacher's whole row / temperature) makes p the teacher's true
    probabilities and adds the mass outside the list as one more event.  The
    mean over the rows (those whose target is not ignore_index, if targets are
    given), or their sum over `denominator`.  Returns loss, losses (of the
    rows), dlogits."""
    if denominator is not None and not denominator > 0:
        raise ValueError(f"denominator must be > 0, not {denominator!r}")
    record = _records(logits, grad)

    def compute():
        rows, shape, device, (b, s), d = _rows(logits, targets, ignore_index, temperature, grad or record, grad_scale, out)
        if not isinstance(teacher_ids, torch.Tensor) or teacher_ids.dim() != len(shape) + 1:
            raise ValueError("teacher_ids must have the logits' dimensions")
        K = teacher_ids.shape[-1]
        lists = shape + (K,)
        ids = _lists(teacher_ids, "teacher_ids", lists, device, _INT)
        t = _lists(teacher_logits, "teacher_logits", lists, device, _ANY)
        lse = _array(teacher_lse, "teacher_lse", shape, device) if teacher_lse is not None else _NONE
        loss = torch.empty((), dtype=torch.float32, device=device)
        losses = torch.empty(shape, dtype=torch.float32, device=device)
        args = _DISTILL_ARGS(K, _ITYPES[teacher_ids.dtype], _DTYPES[teacher_logits.dtype], *ids, *t, *lse, hard_weight,
                             denominator or 0.0, loss.data_ptr(), losses.data_ptr())
        ws, size = _workspace(_DISTILL, rows, b * s, 0, d is not None, device)
        _run("glr_distill_loss", device, rows, args, ws.data_ptr(), size)
        return DistillLoss(loss, losses, d)

    if record:
        return DistillLoss(*_WithGradient.apply(logits, compute), None)
    return compute()
