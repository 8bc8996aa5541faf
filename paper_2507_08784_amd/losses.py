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


_fns = None


def _lib():
    global _fns
    if _fns is None:
        lib = load()
        P = ctypes.POINTER
        sig = {
            "glr_loss_workspace_bytes": [P(Rows), _I32, _I64, P(ctypes.c_size_t)],
            "glr_token_logprobs": [P(Rows), P(RowArray), _VP, _VP, _VP, ctypes.c_size_t, _VP],
            "glr_token_logprobs_backward": [P(Rows), _VP, P(RowArray), _VP],
            "glr_preference_loss": [P(Rows), P(PrefArgs), _VP, ctypes.c_size_t, _VP],
            "glr_policy_loss": [P(Rows), P(PolicyArgs), _VP, ctypes.c_size_t, _VP],
            "glr_distill_loss": [P(Rows), P(DistillArgs), _VP, ctypes.c_size_t, _VP],
            "glr_loss_rescale": [_VP, _I64, _I32, _VP, _VP],
        }
        for name, args in sig.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = _I32, args
        _fns = lib
    return _fns


# ----------------------------------------------------------------------------
# arguments
# ----------------------------------------------------------------------------
_NONE = (None, 0, 0)


def _strides(x, extra=0):
    """(pointer, batch stride, step stride) of an array over the rows."""
    st = x.stride()
    if len(st) - extra == 2:
        return x.data_ptr(), st[0], st[1]
    return x.data_ptr(), 0, st[0]


def _same(x, name, shape, device, dtypes):
    if not torch.is_tensor(x):
        raise TypeError(f"{name} must be a tensor, not {type(x).__name__}")
    if x.dtype not in dtypes:
        raise TypeError(f"{name} must be {' or '.join(str(d) for d in dtypes)}, not {x.dtype}")
    if x.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, not {tuple(x.shape)}")
    if x.device != device:
        raise ValueError(f"{name} must live on {device}, not {x.device}")


_FLOAT = (torch.float32,)
_INT = (torch.int64, torch.int32)
_ANY = (torch.float32, torch.bfloat16, torch.float16)


class _Call:
    """One call's rows: the checks every loss makes, and the C struct."""

    __slots__ = ("logits", "shape", "device", "rows", "dlogits", "keep", "batch", "steps")

    def __init__(self, logits, targets, ignore_index, temperature, grad, grad_scale, out):
        if not torch.is_tensor(logits):
            raise TypeError(f"logits must be a tensor, not {type(logits).__name__}")
        if logits.dtype not in _DTYPES:
            raise TypeError(f"logits must be float32, bfloat16 or float16, not {logits.dtype}")
        if logits.dim() not in (2, 3):
            raise ValueError(f"logits must be (rows, vocab) or (batch, steps, vocab), not {tuple(logits.shape)}")
        if not logits.is_cuda:
            raise ValueError("the losses run on the GPU only (logits on the CPU)")
        shape = logits.shape[:-1]
        device = logits.device
        if logits.shape[-1] > 1 and logits.stride(-1) != 1:
            raise ValueError("a row of logits must be contiguous (stride 1 over the vocabulary)")
        self.logits, self.shape, self.device = logits, shape, device
        if targets is not None:
            _same(targets, "targets", shape, device, _INT)
        d = None
        if out is not None and not grad:
            raise ValueError("out is the gradient's: it needs grad=True (weights=... of token_logprobs)")
        if grad:
            if out is None:
                d = torch.empty(logits.shape, dtype=logits.dtype, device=device)
            else:
                _same(out, "out", logits.shape, device, (logits.dtype,))
                if out.shape[-1] > 1 and out.stride(-1) != 1:
                    raise ValueError("a row of out must be contiguous (stride 1 over the vocabulary)")
                if out.data_ptr() == logits.data_ptr() and out.stride() != logits.stride():
                    raise ValueError("out that replaces the logits must have their strides")
                d = out
        self.dlogits = d
        self.batch, self.steps = (shape[0], shape[1]) if len(shape) == 2 else (1, shape[0])
        self.rows = Rows(self.batch, self.steps, logits.shape[-1], _strides(logits, 1),
                         _strides(d, 1) if d is not None else _NONE, _DTYPES[logits.dtype],
                         _ITYPES[targets.dtype] if targets is not None else 0,
                         _strides(targets) if targets is not None else _NONE, ignore_index, temperature, grad_scale)

    def array(self, x, name, dtypes=_FLOAT):
        _same(x, name, self.shape, self.device, dtypes)
        return _strides(x)

    def lists(self, x, name, shape, dtypes):
        """A per-row list: its last dimension contiguous."""
        _same(x, name, shape, self.device, dtypes)
        if x.shape[-1] > 1 and x.stride(-1) != 1:
            raise ValueError(f"a row of {name} must be contiguous")
        return _strides(x, 1)

    def seqs(self, cu):
        if cu is None:
            if len(self.shape) != 2:
                raise ValueError("packed rows (2-D logits) need cu_seqlens")
            return self.batch, (self.batch, None, 0)
        if cu.dim() != 1 or cu.numel() < 2:
            raise ValueError("cu_seqlens must be one-dimensional with at least two offsets")
        if len(self.shape) != 1:
            raise ValueError("cu_seqlens goes with packed rows (2-D logits)")
        _same(cu, "cu_seqlens", cu.shape, self.device, _INT)
        if not cu.is_contiguous():
            raise ValueError("cu_seqlens must be contiguous")
        n = cu.numel() - 1
        return n, (n, cu.data_ptr(), _ITYPES[cu.dtype])

    def f32(self, *shape):
        return torch.empty(shape, dtype=torch.float32, device=self.device)

    def workspace(self, op, seqs):
        n = ctypes.c_size_t()
        _check(_lib().glr_loss_workspace_bytes(self.rows, op, seqs, n))
        return torch.empty(n.value, dtype=torch.uint8, device=self.device), n.value

    def run(self, fn, *args):
        dev = self.device
        if dev.index != torch.cuda.current_device():
            with torch.cuda.device(dev):
                _check(fn(*args, torch.cuda.current_stream(dev).cuda_stream))
        else:
            _check(fn(*args, torch.cuda.current_stream(dev).cuda_stream))


def _records(logits, grad):
    """Whether a call is part of the graph (and not an explicit one)."""
    return not grad and torch.is_tensor(logits) and logits.requires_grad and torch.is_grad_enabled()


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
        rest = tuple(x for x in result[1:-1])
        ctx.mark_non_differentiable(*rest)
        return (result.loss,) + rest

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_loss, *_):
        d, ctx.dlogits = ctx.dlogits, None
        if d is None:
            raise RuntimeError("the loss's gradient was handed on already: call the loss again for a second backward")
        scale = grad_loss.float().contiguous()
        dev = d.device
        with torch.cuda.device(dev):
            _check(_lib().glr_loss_rescale(d.data_ptr(), d.numel(), _DTYPES[d.dtype], scale.data_ptr(),
                                           torch.cuda.current_stream(dev).cuda_stream))
        return d, None


class _TokenLogprobs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, targets, temperature, ignore_index):
        c = _Call(logits, targets, ignore_index, temperature, False, 1.0, None)
        logps, stats = c.f32(*c.shape), c.f32(c.batch * c.steps, 2)
        c.run(_lib().glr_token_logprobs, c.rows, None, logps.data_ptr(), stats.data_ptr(), None, 0)
        ctx.save_for_backward(logits, targets, stats)
        ctx.options = (ignore_index, temperature)
        return logps

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad):
        logits, targets, stats = ctx.saved_tensors
        ignore_index, temperature = ctx.options
        c = _Call(logits, targets, ignore_index, temperature, True, 1.0, None)
        w = RowArray(*c.array(grad, "the upstream gradient"))
        c.run(_lib().glr_token_logprobs_backward, c.rows, stats.data_ptr(), w)
        return c.dlogits, None, None, None


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
    c = _Call(logits, targets, ignore_index, temperature, weights is not None, grad_scale, out)
    w = RowArray(*c.array(weights, "weights")) if weights is not None else None
    logps = c.f32(*c.shape)
    c.run(_lib().glr_token_logprobs, c.rows, w, logps.data_ptr(), None, None, 0)
    return TokenLogprobs(logps, c.dlogits)


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
        c = _Call(logits, targets, ignore_index, 1.0, grad or record, grad_scale, out)
        n, seqs = c.seqs(cu_seqlens)
        _same(ref_logps, "ref_logps", (n,), c.device, _FLOAT)
        if not ref_logps.is_contiguous():
            raise ValueError("ref_logps must be contiguous")
        loss, logps, rewards = c.f32(), c.f32(n), c.f32(n)
        args = PrefArgs(seqs, KINDS[kind], bool(average), beta, label_smoothing, ref_logps.data_ptr(),
                        loss.data_ptr(), logps.data_ptr(), rewards.data_ptr())
        ws, size = c.workspace(_PREFERENCE, n)
        c.run(_lib().glr_preference_loss, c.rows, args, ws.data_ptr(), size)
        return PreferenceLoss(loss, logps, rewards, c.dlogits)

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
        c = _Call(logits, targets, ignore_index, temperature, grad or record, grad_scale, out)
        n, seqs = 0, (0, None, 0)
        if cu_seqlens is not None or reduction == "sequence":
            n, seqs = c.seqs(cu_seqlens)
        old, adv = c.array(old_logps, "old_logps"), c.array(advantages, "advantages")
        ref = c.array(ref_logps, "ref_logps") if ref_logps is not None else _NONE
        loss, kl, clipped, logps = c.f32(), c.f32(), c.f32(), c.f32(*c.shape)
        args = PolicyArgs(seqs, REDUCTIONS[reduction], clip_low, clip_high, kl_coef, denominator or 0.0, old, adv, ref,
                          loss.data_ptr(), kl.data_ptr(), clipped.data_ptr(), logps.data_ptr())
        ws, size = c.workspace(_POLICY, n)
        c.run(_lib().glr_policy_loss, c.rows, args, ws.data_ptr(), size)
        return PolicyLoss(loss, logps, kl, clipped, c.dlogits)

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
        c = _Call(logits, targets, ignore_index, temperature, grad or record, grad_scale, out)
        if not torch.is_tensor(teacher_ids) or teacher_ids.dim() != len(c.shape) + 1:
            raise ValueError("teacher_ids must have the logits' dimensions")
        K = teacher_ids.shape[-1]
        shape = c.shape + (K,)
        ids = c.lists(teacher_ids, "teacher_ids", shape, _INT)
        t = c.lists(teacher_logits, "teacher_logits", shape, _ANY)
        lse = c.array(teacher_lse, "teacher_lse") if teacher_lse is not None else _NONE
        loss, losses = c.f32(), c.f32(*c.shape)
        args = DistillArgs(K, _ITYPES[teacher_ids.dtype], _DTYPES[teacher_logits.dtype], ids, t, lse, hard_weight,
                           denominator or 0.0, loss.data_ptr(), losses.data_ptr())
        ws, size = c.workspace(_DISTILL, 0)
        c.run(_lib().glr_distill_loss, c.rows, args, ws.data_ptr(), size)
        return DistillLoss(loss, losses, c.dlogits)

    if record:
        return DistillLoss(*_WithGradient.apply(logits, compute), None)
    return compute()
