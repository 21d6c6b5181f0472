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
import functools

import torch

from . import binding as B

__all__ = ["token_logprob", "token_logprob_grad", "preference_loss", "policy_loss", "balance_loss"]

_TYPES = {torch.float32: B.F32, torch.bfloat16: B.BF16}

# A call on few rows lasts as long as its marshalling: the current stream's
# handle is asked for directly (torch.cuda.current_stream takes 2 us) and sizes are
# kept.  Every output has a storage of its own (1.4 us each; a view of a common one 0.9), so
# that a loss that is kept keeps no workspace.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _address(t):
    return None if t is None else t.data_ptr()


def _vector(name, t, dtype, shape, device):
    """Refuses what is not a contiguous tensor of that type and shape on that device."""
    try:
        if t.dtype is dtype and t.shape == shape and t.device == device and t.is_contiguous():
            return
    except AttributeError:
        pass
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, the logits are on {device}")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, not {t.dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, not {tuple(t.shape)}")
    raise ValueError(f"{name} must be contiguous")


def _matrix(name, t):
    """(rows, classes, pitch) of a tensor whose rows are contiguous."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if t.dim() != 2 or t.dtype not in _TYPES:
        raise ValueError(f"{name} must be [rows, classes] in float32 or bfloat16")
    rows, classes = t.shape
    pitch, step = t.stride()
    if classes < 1:
        raise ValueError(f"{name} must have a class")
    if classes > 1 and step != 1:
        raise ValueError(f"rows of {name} must be contiguous")
    if rows < 2:
        return rows, classes, classes
    if pitch < classes:
        raise ValueError(f"rows of {name} overlap")
    return rows, classes, pitch


def _gradient(logits, out, grad):
    """The tensor for the gradient and its pitch."""
    if not grad:
        if out is not None:
            raise ValueError("out was given for a gradient that is not asked for")
        return None, 0
    if out is None:
        rows, classes = logits.shape
        return torch.empty((rows, classes), dtype=logits.dtype, device=logits.device), classes
    pitch = _matrix("out", out)[2]
    if out.shape != logits.shape or out.dtype != logits.dtype or out.device != logits.device:
        raise ValueError("out must have the logits' shape, type and device")
    return out, pitch


def _on(device, stream, tensors, call):
    """call(stream handle) with the device and stream current; tensors given
    are kept from reuse until a stream that is not current is past the call."""
    if stream is None and device.index == torch.cuda.current_device():
        return call(_raw_stream(device.index))
    if stream is None:
        stream = torch.cuda.current_stream(device)
    elif not hasattr(stream, "cuda_stream"):
        stream = torch.cuda.ExternalStream(int(stream), device=device) if int(stream) else \
            torch.cuda.default_stream(device)
    if stream.device != device:
        raise ValueError(f"the stream is on {stream.device}, the logits are on {device}")
    with torch.cuda.stream(stream):
        result = call(stream.cuda_stream)
    for t in tensors:
        if t is not None:
            t.record_stream(stream)
    return result


@functools.lru_cache(maxsize=4096)
def _bytes(query, *sizes):
    n = C.c_int64()
    B._check(getattr(B.lib, query)(*sizes, C.byref(n)), query)
    return n.value


def token_logprob(logits, target, temperature=1.0, *, stream=None):
    """Log probability of every row's target (float32 [rows], 0 without one), and the rows'
    statistics (float32 [rows, 2]) that ``token_logprob_grad`` takes."""
    rows, classes, ld = _matrix("logits", logits)
    device = logits.device
    _vector("target", target, torch.int32, (rows,), device)

    def call(st):
        logp = torch.empty(rows, dtype=torch.float32, device=device)
        stats = torch.empty((rows, 2), dtype=torch.float32, device=device)
        z = B.Logits(logits.data_ptr(), target.data_ptr(), None, rows, classes, ld, 0, _TYPES[logits.dtype], temperature)
        B._check(B.lib.pgc_token_logprob(z, logp.data_ptr(), stats.data_ptr(), st), "pgc_token_logprob")
        return logp, stats
    return _on(device, stream, (logits, target), call)


def token_logprob_grad(logits, target, stats, dlogp, temperature=1.0, *, out=None, stream=None):
    """Gradient of the logits for the derivatives dlogp (float32 [rows]) of a loss with
    respect to the rows' log probabilities."""
    rows, classes, ld = _matrix("logits", logits)
    device = logits.device
    _vector("target", target, torch.int32, (rows,), device)
    _vector("stats", stats, torch.float32, (rows, 2), device)
    _vector("dlogp", dlogp, torch.float32, (rows,), device)

    def call(st):
        dlogits, ldg = _gradient(logits, out, True)
        z = B.Logits(logits.data_ptr(), target.data_ptr(), dlogits.data_ptr(), rows, classes, ld, ldg,
                     _TYPES[logits.dtype], temperature)
        B._check(B.lib.pgc_token_logprob_grad(z, stats.data_ptr(), dlogp.data_ptr(), st), "pgc_token_logprob_grad")
        return dlogits
    return _on(device, stream, (logits, target, stats, dlogp, out), call)


def preference_loss(logits, target, offsets, ref_logp=None, *, beta=0.1, kind="sigmoid", margin=0.0, smoothing=0.0,
                    average=False, scale=1.0, temperature=1.0, grad=True, out=None, stream=None):
    """Preference loss of pairs of sequences: sequence 2 i, rows offsets[2 i] to
    offsets[2 i + 1], is preferred to sequence 2 i + 1.

    offsets is int32 [2 pairs + 1], ref_logp float32 [pairs, 2] (the reference's scores), kind
    "sigmoid", "hinge" or "squared".  Returns a dict: loss (scalar), logp (float32
    [pairs, 2], the sequences' scores), dlogits.
    """
    rows, classes, ld = _matrix("logits", logits)
    device = logits.device
    _vector("target", target, torch.int32, (rows,), device)
    n = offsets.numel() if isinstance(offsets, torch.Tensor) else 0
    _vector("offsets", offsets, torch.int32, (n,), device)
    if n % 2 == 0:
        raise ValueError("offsets must have 2 pairs + 1 entries")
    pairs = n // 2
    if ref_logp is not None:
        _vector("ref_logp", ref_logp, torch.float32, (pairs, 2), device)
    kind = B._enum(kind, B.PREFERENCES)

    def call(st):
        dlogits, ldg = _gradient(logits, out, grad)
        size = _bytes("pgc_loss_workspace", rows, 2 * pairs)
        loss = torch.empty((), dtype=torch.float32, device=device)
        logp = torch.empty((pairs, 2), dtype=torch.float32, device=device)
        ws = torch.empty(size, dtype=torch.uint8, device=device)
        z = B.Logits(logits.data_ptr(), target.data_ptr(), _address(dlogits), rows, classes, ld, ldg,
                     _TYPES[logits.dtype], temperature)
        B._check(B.lib.pgc_preference_loss(z, kind, pairs, offsets.data_ptr(), _address(ref_logp), beta, margin,
                                           smoothing, 1 if average else 0, scale, loss.data_ptr(), logp.data_ptr(),
                                           ws.data_ptr(), size, st), "pgc_preference_loss")
        return {"loss": loss, "logp": logp, "dlogits": dlogits}
    return _on(device, stream, (logits, target, offsets, ref_logp, out), call)


def policy_loss(logits, target, old_logp, advantage, ref_logp=None, *, clip=(0.2, 0.2), kl=0.0, offsets=None,
                reduction="tokens", scale=1.0, temperature=1.0, grad=True, out=None, stream=None):
    """Clipped policy loss with a KL term, over rows of sampled tokens.

    old_logp, advantage, ref_logp are float32 [rows]; clip = (below, above) 1; reduction
    "tokens", "sequences" (needs offsets, int32 [sequences + 1]) or "sum".  Returns a
    dict: loss (scalar), terms (float32 [3]: policy term, KL, clipped share), logp
    (float32 [rows]), dlogits.
    """
    rows, classes, ld = _matrix("logits", logits)
    device = logits.device
    _vector("target", target, torch.int32, (rows,), device)
    _vector("old_logp", old_logp, torch.float32, (rows,), device)
    _vector("advantage", advantage, torch.float32, (rows,), device)
    if ref_logp is not None:
        _vector("ref_logp", ref_logp, torch.float32, (rows,), device)
    reduction = B._enum(reduction, B.REDUCTIONS)
    sequences = 0
    if reduction == B.REDUCTIONS["sequences"]:
        if not isinstance(offsets, torch.Tensor) or offsets.numel() < 1:
            raise ValueError('reduction "sequences" needs offsets')
        sequences = offsets.numel() - 1
        _vector("offsets", offsets, torch.int32, (sequences + 1,), device)
    elif offsets is not None:
        raise ValueError('offsets go with reduction "sequences"')
    low, high = clip

    def call(st):
        dlogits, ldg = _gradient(logits, out, grad)
        size = _bytes("pgc_loss_workspace", rows, sequences)
        loss = torch.empty((), dtype=torch.float32, device=device)
        terms = torch.empty(3, dtype=torch.float32, device=device)
        logp = torch.empty(rows, dtype=torch.float32, device=device)
        ws = torch.empty(size, dtype=torch.uint8, device=device)
        z = B.Logits(logits.data_ptr(), target.data_ptr(), _address(dlogits), rows, classes, ld, ldg,
                     _TYPES[logits.dtype], temperature)
        B._check(B.lib.pgc_policy_loss(z, reduction, sequences, _address(offsets), old_logp.data_ptr(),
                                       advantage.data_ptr(), _address(ref_logp), low, high, kl, scale, loss.data_ptr(),
                                       terms.data_ptr(), logp.data_ptr(), ws.data_ptr(), size, st), "pgc_policy_loss")
        return {"loss": loss, "terms": terms, "logp": logp, "dlogits": dlogits}
    return _on(device, stream, (logits, target, old_logp, advantage, ref_logp, offsets, out), call)


def balance_loss(logits, k, *, mask=None, choice=None, alpha=0.01, grad=True, out=None, stream=None):
    """A router's choice of k experts per token, its counts and its balance loss.

    logits is [tokens, experts]; mask uint8 [tokens], 0 for padding; choice int32 [tokens, k]
    if the router chose otherwise than by its largest logits (it is then only
    counted).  Returns a dict: loss (scalar), counts (int32 [experts]), choice, dlogits.
    """
    rows, experts, ld = _matrix("logits", logits)
    device = logits.device
    if mask is not None:
        _vector("mask", mask, torch.uint8, (rows,), device)
    given = choice is not None
    if given:
        _vector("choice", choice, torch.int32, (rows, k), device)
    size = _bytes("pgc_balance_workspace", rows, experts)

    def call(st):
        dlogits, ldg = _gradient(logits, out, grad)
        loss = torch.empty((), dtype=torch.float32, device=device)
        counts = torch.empty(experts, dtype=torch.int32, device=device)
        chosen = choice if given else torch.empty((rows, max(k, 0)), dtype=torch.int32, device=device)
        ws = torch.empty(size, dtype=torch.uint8, device=device)
        B._check(B.lib.pgc_balance_loss(_TYPES[logits.dtype], rows, experts, logits.data_ptr(), ld, _address(mask), k,
                                        1 if given else 0, chosen.data_ptr(), alpha, loss.data_ptr(),
                                        counts.data_ptr(), _address(dlogits), ldg, ws.data_ptr(), size, st),
                 "pgc_balance_loss")
        return {"loss": loss, "counts": counts, "choice": chosen, "dlogits": dlogits}
    return _on(device, stream, (logits, mask, choice, out), call)
