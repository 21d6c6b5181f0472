"""Losses on rows of logits with their gradients, for torch CUDA tensors.

Thin layer over the calls of include/pgc.h that take a caller's logits: it
checks shapes and types, allocates outputs and workspace through torch's
allocator, and passes pointers.  Each function returns a loss together with its
gradient with respect to the logits (``dlogits``, of the logits' type), which a
model's own backward pass starts from; nothing here is recorded by autograd.

Common arguments:
  logits       [rows, classes] float32 or bfloat16, rows contiguous (any row pitch)
  target       [rows] int32, negative: the row takes no part
  temperature  the logits are divided by it
  out          tensor for dlogits (shaped and typed as logits; may be logits itself)
  grad         False: the loss alone, no dlogits
  stream       torch stream or cudaStream_t; default: torch's current stream of
               the tensors' device.  Outputs and workspace are allocated for that
               stream; tensors given must be ready on it
"""

from __future__ import annotations

import ctypes as C

import torch

from . import binding as B

__all__ = ["token_logprob", "token_logprob_grad", "preference_loss", "policy_loss", "balance_loss"]

_TYPES = {torch.float32: B.F32, torch.bfloat16: B.BF16}


def _address(t):
    return None if t is None else t.data_ptr()


def _vector(name, t, dtype, shape, device, optional=False):
    """A contiguous tensor of that type and shape on that device."""
    if t is None and optional:
        return None
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, the logits are on {device}")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, not {t.dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, not {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t


def _matrix(name, t):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if t.dim() != 2 or t.dtype not in _TYPES:
        raise ValueError(f"{name} must be [rows, classes] in float32 or bfloat16")
    if t.shape[1] < 1:
        raise ValueError(f"{name} must have a class")
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"rows of {name} must be contiguous")
    return t


def _pitch(name, t):
    """Elements between rows."""
    if t.shape[0] < 2:
        return t.shape[1]
    if t.stride(0) < t.shape[1]:
        raise ValueError(f"rows of {name} overlap")
    return t.stride(0)


def _gradient(logits, out, grad):
    if not grad:
        if out is not None:
            raise ValueError("out was given for a gradient that is not asked for")
        return None
    if out is None:
        return torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
    _matrix("out", out)
    if out.shape != logits.shape or out.dtype != logits.dtype or out.device != logits.device:
        raise ValueError("out must have the logits' shape, type and device")
    return out


class _On:
    """Makes a device and stream current for a call, where they are not already."""

    def __init__(self, device, stream):
        current = torch.cuda.current_stream(device)
        if stream is None:
            stream = current
        elif not hasattr(stream, "cuda_stream"):
            stream = torch.cuda.ExternalStream(int(stream), device=device) if int(stream) else \
                torch.cuda.default_stream(device)
        if stream.device != device:
            raise ValueError(f"the stream is on {stream.device}, the logits are on {device}")
        self.handle = stream.cuda_stream
        same = stream == current and torch.cuda.current_device() == device.index
        self._guard = None if same else torch.cuda.stream(stream)

    def __enter__(self):
        if self._guard is not None:
            self._guard.__enter__()
        return self.handle

    def __exit__(self, *exc):
        if self._guard is not None:
            self._guard.__exit__(*exc)


def _rows(logits, target, temperature, dlogits):
    return B.Logits(logits.data_ptr(), target.data_ptr(), _address(dlogits), logits.shape[0], logits.shape[1],
                    _pitch("logits", logits), _pitch("out", dlogits) if dlogits is not None else 0,
                    _TYPES[logits.dtype], temperature)


def _workspace(size, device, *args):
    n = C.c_int64()
    B._check(size(*args, C.byref(n)), "workspace size")
    return torch.empty(n.value, dtype=torch.uint8, device=device)


def token_logprob(logits, target, temperature=1.0, *, stream=None):
    """Log probability of every row's target (float32 [rows], 0 without one), and the rows'
    statistics (float32 [rows, 2]) that ``token_logprob_grad`` takes."""
    _matrix("logits", logits)
    rows, device = logits.shape[0], logits.device
    _vector("target", target, torch.int32, (rows,), device)
    with _On(device, stream) as st:
        logp = torch.empty(rows, dtype=torch.float32, device=device)
        stats = torch.empty((rows, 2), dtype=torch.float32, device=device)
        z = _rows(logits, target, temperature, None)
        B._check(B.lib.pgc_token_logprob(C.byref(z), logp.data_ptr(), stats.data_ptr(), st), "pgc_token_logprob")
    return logp, stats


def token_logprob_grad(logits, target, stats, dlogp, temperature=1.0, *, out=None, stream=None):
    """Gradient of the logits for the derivatives dlogp (float32 [rows]) of a loss with
    respect to the rows' log probabilities."""
    _matrix("logits", logits)
    rows, device = logits.shape[0], logits.device
    _vector("target", target, torch.int32, (rows,), device)
    _vector("stats", stats, torch.float32, (rows, 2), device)
    _vector("dlogp", dlogp, torch.float32, (rows,), device)
    with _On(device, stream) as st:
        dlogits = _gradient(logits, out, True)
        z = _rows(logits, target, temperature, dlogits)
        B._check(B.lib.pgc_token_logprob_grad(C.byref(z), stats.data_ptr(), dlogp.data_ptr(), st),
                 "pgc_token_logprob_grad")
    return dlogits


def preference_loss(logits, target, offsets, ref_logp=None, *, beta=0.1, kind="sigmoid", margin=0.0, smoothing=0.0,
                    average=False, scale=1.0, temperature=1.0, grad=True, out=None, stream=None):
    """Preference loss of pairs of sequences: sequence 2 i, rows offsets[2 i] to
    offsets[2 i + 1], is preferred to sequence 2 i + 1.

    offsets is int32 [2 pairs + 1], ref_logp float32 [pairs, 2] (the reference's scores), kind
    "sigmoid", "hinge" or "squared".  Returns a dict: loss (scalar), logp (float32
    [pairs, 2], the sequences' scores), dlogits.
    """
    _matrix("logits", logits)
    rows, device = logits.shape[0], logits.device
    _vector("target", target, torch.int32, (rows,), device)
    n = offsets.numel() if isinstance(offsets, torch.Tensor) else 0
    _vector("offsets", offsets, torch.int32, (n,), device)
    if n % 2 == 0:
        raise ValueError("offsets must have 2 pairs + 1 entries")
    pairs = n // 2
    _vector("ref_logp", ref_logp, torch.float32, (pairs, 2), device, optional=True)
    with _On(device, stream) as st:
        dlogits = _gradient(logits, out, grad)
        loss = torch.empty((), dtype=torch.float32, device=device)
        logp = torch.empty((pairs, 2), dtype=torch.float32, device=device)
        ws = _workspace(B.lib.pgc_loss_workspace, device, rows, 2 * pairs)
        z = _rows(logits, target, temperature, dlogits)
        B._check(B.lib.pgc_preference_loss(C.byref(z), B._enum(kind, B.PREFERENCES), pairs, offsets.data_ptr(),
                                           _address(ref_logp), beta, margin, smoothing, 1 if average else 0, scale,
                                           loss.data_ptr(), logp.data_ptr(), ws.data_ptr(), ws.numel(), st),
                 "pgc_preference_loss")
    return {"loss": loss, "logp": logp, "dlogits": dlogits}


def policy_loss(logits, target, old_logp, advantage, ref_logp=None, *, clip=(0.2, 0.2), kl=0.0, offsets=None,
                reduction="tokens", scale=1.0, temperature=1.0, grad=True, out=None, stream=None):
    """Clipped policy loss with a KL term, over rows of sampled tokens.

    old_logp, advantage, ref_logp are float32 [rows]; clip = (below, above) 1; reduction
    "tokens", "sequences" (needs offsets, int32 [sequences + 1]) or "sum".  Returns a
    dict: loss (scalar), terms (float32 [3]: policy term, KL, clipped share), logp
    (float32 [rows]), dlogits.
    """
    _matrix("logits", logits)
    rows, device = logits.shape[0], logits.device
    _vector("target", target, torch.int32, (rows,), device)
    _vector("old_logp", old_logp, torch.float32, (rows,), device)
    _vector("advantage", advantage, torch.float32, (rows,), device)
    _vector("ref_logp", ref_logp, torch.float32, (rows,), device, optional=True)
    sequences = 0
    if B._enum(reduction, B.REDUCTIONS) == B.REDUCTIONS["sequences"]:
        if not isinstance(offsets, torch.Tensor) or offsets.numel() < 1:
            raise ValueError('reduction "sequences" needs offsets')
        sequences = offsets.numel() - 1
        _vector("offsets", offsets, torch.int32, (sequences + 1,), device)
    elif offsets is not None:
        raise ValueError('offsets go with reduction "sequences"')
    with _On(device, stream) as st:
        dlogits = _gradient(logits, out, grad)
        small = torch.empty(4, dtype=torch.float32, device=device)
        logp = torch.empty(rows, dtype=torch.float32, device=device)
        ws = _workspace(B.lib.pgc_loss_workspace, device, rows, sequences)
        z = _rows(logits, target, temperature, dlogits)
        B._check(B.lib.pgc_policy_loss(C.byref(z), B._enum(reduction, B.REDUCTIONS), sequences, _address(offsets),
                                       old_logp.data_ptr(), advantage.data_ptr(), _address(ref_logp), clip[0], clip[1],
                                       kl, scale, small.data_ptr(), small.data_ptr() + 4, logp.data_ptr(),
                                       ws.data_ptr(), ws.numel(), st), "pgc_policy_loss")
    return {"loss": small[0], "terms": small[1:], "logp": logp, "dlogits": dlogits}


def balance_loss(logits, k, *, mask=None, choice=None, alpha=0.01, grad=True, out=None, stream=None):
    """A router's choice of k experts per token, its counts and its balance loss.

    logits is [tokens, experts]; mask uint8 [tokens], 0 for padding; choice int32 [tokens, k]
    if the router chose otherwise than by its largest logits (it is then only
    counted).  Returns a dict: loss (scalar), counts (int32 [experts]), choice, dlogits.
    """
    _matrix("logits", logits)
    (rows, experts), device = logits.shape, logits.device
    _vector("mask", mask, torch.uint8, (rows,), device, optional=True)
    given = choice is not None
    if given:
        _vector("choice", choice, torch.int32, (rows, k), device)
    with _On(device, stream) as st:
        dlogits = _gradient(logits, out, grad)
        loss = torch.empty((), dtype=torch.float32, device=device)
        counts = torch.empty(experts, dtype=torch.int32, device=device)
        if not given:
            choice = torch.empty((rows, max(int(k), 0)), dtype=torch.int32, device=device)
        ws = _workspace(B.lib.pgc_balance_workspace, device, rows, experts)
        B._check(B.lib.pgc_balance_loss(_TYPES[logits.dtype], rows, experts, logits.data_ptr(),
                                        _pitch("logits", logits), _address(mask), k, 1 if given else 0,
                                        choice.data_ptr(), alpha, loss.data_ptr(), counts.data_ptr(),
                                        _address(dlogits), _pitch("out", dlogits) if dlogits is not None else 0,
                                        ws.data_ptr(), ws.numel(), st), "pgc_balance_loss")
    return {"loss": loss, "counts": counts, "choice": choice, "dlogits": dlogits}
