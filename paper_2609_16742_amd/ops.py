"""The operators around a protected classifier, on torch tensors.

Group norm with an activation on channels-last maps (``group_norm``), 8-bit
matrices with a scale for each block of 128 (``fp8_quantize``) and their
product (``fp8_matmul``), and the scores of given classes or tokens
(``token_scores``), with the backward passes of the first and the last; for a
head over a map's pixels, attention (``attention``), the norms and rotations
of its queries and keys (``head_norm_rotary``), both with their backward
passes, and the clipping of all gradients by their norm (``clip_gradients``).
Checks of arguments, outputs and workspaces (csrc/binding.cpp); the work runs
in libctc.so's HIP kernels (include/ctc.h states what each computes).

Every call takes tensors of one GPU, enqueues on ``stream`` (default: the
current stream of that GPU) and returns without waiting.  Outputs are
allocated unless given, as that stream's tensors (as under
``torch.cuda.stream``): work on another stream that reads them has to wait for
it and call ``record_stream``.  Inputs have to outlive their use there.  Nothing
is recorded for autograd: the backward passes are calls of their own, and
tensors that require grad are refused unless under ``torch.no_grad()``.  Wrong
shapes, types or devices raise ValueError before anything is enqueued; the
library's own refusals raise :class:`ctc.CtcError`.
"""

from __future__ import annotations

from typing import NamedTuple, Optional

import torch

from . import ctc

try:
    from . import _binding
except ImportError as e:
    raise ImportError(
        "the operators' binding is not built (%s); run __graft_entry__.build()"
        " or python paper_2609_16742_amd/build.py" % e) from e

_binding.set_check(ctc._check)

_ACT = {"none": ctc.CTC_ACT_NONE, "relu": ctc.CTC_ACT_RELU,
        "silu": ctc.CTC_ACT_SILU}
_QTYPE = {"e4m3": False, "e5m2": True}

_current_raw = torch._C._cuda_getCurrentRawStream


def _act(act):
    try:
        return _ACT[act]
    except (KeyError, TypeError):
        raise ValueError("act must be one of %s" % sorted(_ACT)) from None


def _run(f, t, stream, *args):
    """f(*args, raw stream) on ``stream`` (None: the current one) of t's GPU.
    Outputs and workspaces are allocated with that stream current: a block
    of another stream's could still be in use there."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda):
        raise ValueError("GPU tensors are needed")
    current = _current_raw(t.get_device())
    if stream is None:
        return f(*args, current)
    raw = stream if isinstance(stream, int) else stream.cuda_stream
    if raw == current:
        return f(*args, raw)
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(raw, device=t.device)
    if stream.device != t.device:
        raise ValueError("the stream is another GPU's")
    with torch.cuda.stream(stream):
        return f(*args, raw)


def group_norm(x, groups, gamma=None, beta=None, residual=None, act="none",
               carry=False, eps=1e-5, out=None, stream=None):
    """y, mean, rstd of a channels-last map ``x`` [n, ..., c]:
    ``y = act((x - mean) * rstd * gamma + beta (+ residual))`` with
    statistics over each image's pixels and each of ``groups`` channel groups
    (mean and rstd [n, groups], fp32).  ``act`` is "none", "relu" or "silu".
    With ``carry`` the last channel is a carry-through checksum, which takes
    no part and passes (plus the residual's).  ``out``: a (y, mean, rstd) of
    an earlier call to write into; its y may be x or residual."""
    y, mean, rstd = out or (None, None, None)
    return _run(_binding.group_norm, x, stream, x, groups, gamma, beta,
                residual, _act(act), carry, eps, y, mean, rstd)


def group_norm_backward(dy, x, mean, rstd, groups, gamma=None, beta=None,
                        residual=None, act="none", carry=False, out=None,
                        stream=None):
    """dx, dresidual, dgamma, dbeta of :func:`group_norm` (same arguments,
    with the ``mean`` and ``rstd`` it returned); dresidual is None without a
    residual, dgamma and dbeta are always given (fp32).  ``out``: a tuple of
    an earlier call to write into, or of tensors and None (not wanted); its
    dx or its dresidual may be dy."""
    dx, dr, dgamma, dbeta = out or (None, None, None, None)
    return _run(_binding.group_norm_backward, x, stream, dy, x, mean, rstd,
                groups, gamma, beta, residual, _act(act), carry, out is None,
                dx, dr, dgamma, dbeta)


def fp8_quantize(x, qtype="e4m3", block_rows=1, transpose=False, out=None,
                 stream=None):
    """(q, scales) of a matrix: ``x`` (or its transpose) in 8 bits ("e4m3" or
    "e5m2") with a scale for each ``block_rows`` (1 or 128) rows by 128
    columns.  q is a float8 tensor whose rows begin at multiples of 16 bytes,
    scales [column blocks, row blocks] fp32; x is about q * scale."""
    if qtype not in _QTYPE:
        raise ValueError("qtype must be one of %s" % sorted(_QTYPE))
    q, scales = out or (None, None)
    return _run(_binding.fp8_quantize, x, stream, x, _QTYPE[qtype],
                block_rows, transpose, q, scales)


def fp8_matmul(a, a_scales, b, b_scales, bias=None, act="none",
               dtype=torch.float16, out=None, stream=None):
    """act(A @ B.T + bias) in ``dtype`` for 8-bit matrices a [m, k] and
    b [n, k] with the scales of :func:`fp8_quantize` (A and B are the values
    they stand for).  16-bit results come of the matrix unit's 8-bit sums,
    which drop of each eight products what lies 13 bits below the largest;
    float32 results, to be rounded afterwards if need be, of fp32 sums."""
    return _run(_binding.fp8_matmul, a, stream, a, a_scales, b, b_scales,
                bias, _act(act), dtype, out)


class TokenScores(NamedTuple):
    """Scores of rows of logits (fp32, int32): see :func:`token_scores`."""
    lse: torch.Tensor
    entropy: torch.Tensor
    logprob: Optional[torch.Tensor]
    rank: Optional[torch.Tensor]
    top_ids: Optional[torch.Tensor]
    top_logprobs: Optional[torch.Tensor]


_NO_SCORES = (None,) * 6


def token_scores(logits, targets=None, top_k=0, out=None, stream=None):
    """Scores of ``logits`` [rows, vocab] (rows may be strided: a protected
    classifier's ``out[:, :classes]``): log-sum-exp, entropy in nats, and for
    int32 ``targets`` [rows] (negative: none) the log probability and the
    rank, and the ``top_k`` best alternatives with their log probabilities
    (ties to the lower index; -1 and -inf where there is none).  ``out``: a
    TokenScores of an earlier call to write into."""
    return TokenScores._make(_run(
        _binding.token_scores, logits, stream, logits, targets, top_k,
        out is None, out or _NO_SCORES))


def token_scores_backward(logits, targets, lse, entropy=None, g_lse=None,
                          g_logprob=None, g_entropy=None, out=None,
                          stream=None):
    """Gradient of the scores' lse, logprob and entropy with respect to the
    logits, given those of the loss with respect to them (each [rows] fp32 or
    None).  ``out`` may be logits itself."""
    if lse is None:
        raise ValueError("lse is needed")
    return _run(_binding.token_scores_backward, logits, stream, logits,
                targets, lse, entropy, g_lse, g_logprob, g_entropy, out)


def attention(q, k, v, causal=False, q_lengths=None, k_lengths=None,
              scale=None, out=None, stream=None):
    """(o, lse) of queries ``q`` [batch, tokens, heads, head size] over keys
    and values ``k``, ``v`` [batch, keys, key heads, head size], float16 or
    bfloat16, head sizes multiples of 8 up to 128, strided as a projection's
    parts are: ``o = softmax(scale q k^T) v`` (``scale``: default 1 /
    sqrt(head size)) and the rows' log-sum-exp [batch, heads, tokens].  Each
    key head serves heads / key heads query heads.  ``q_lengths`` and
    ``k_lengths`` (int32 [batch]): what stands behind them takes no part.
    With ``causal``, query i sees keys up to i + keys - queries (of the
    sequence's own).  A query that sees nothing has o = 0, lse = -inf.
    ``out``: an (o, lse) to write into; o may be q, but overlaps no other
    input."""
    o, lse = out or (None, None)
    return _run(_binding.attention, q, stream, q, k, v, causal, q_lengths,
                k_lengths, scale, o, lse)


def attention_backward(do, q, k, v, o, lse, causal=False, q_lengths=None,
                       k_lengths=None, scale=None, out=None, stream=None):
    """dq, dk, dv of :func:`attention` (same arguments, with the ``o`` and
    ``lse`` it returned) for the gradient ``do`` of o.  Probabilities are
    computed again.  ``out``: a (dq, dk, dv) to write into, which may be parts
    of one projection's gradient; dk and dv may be k or v, but no other input
    and not each other is overlapped."""
    dq, dk, dv = out or (None, None, None)
    return _run(_binding.attention_backward, q, stream, do, q, k, v, o, lse,
                causal, q_lengths, k_lengths, scale, dq, dk, dv)


def grid_positions(*sizes, device="cuda"):
    """int32 [tokens, axes] positions of a grid's points in the order of a
    flattened map: ``grid_positions(h, w)``, ``grid_positions(frames, h,
    w)``."""
    grid = torch.meshgrid(*[torch.arange(n, dtype=torch.int32, device=device)
                            for n in sizes], indexing="ij")
    return torch.stack([g.flatten() for g in grid], 1).contiguous()


def rotary_frequencies(axes, base=10000.0, device="cuda"):
    """fp32 frequencies of ``axes`` (pairs of each): base ** (-i / pairs) for
    pair i of each axis."""
    return torch.cat([torch.empty(0, device=device)] + [
        (base ** (-torch.arange(n, dtype=torch.float64, device=device) / n))
        .float() for n in axes if n])


def head_norm_rotary(q, k=None, q_weight=None, k_weight=None, positions=None,
                     frequencies=None, axes=(), interleaved=False, norm=True,
                     eps=1e-6, dtype=None, out=None, stream=None):
    """(q', k'): the RMS norm of each head of ``q`` and ``k`` [batch, tokens,
    heads, head size] times their weights (fp32 [head size]) and the rotation
    of each head's pairs by their positions.  ``axes`` are the pairs turned
    by each position axis, in order; ``positions`` int32 [tokens, axes] or
    [batch, tokens, axes]; ``frequencies`` fp32, one a pair, in radians a step
    (:func:`grid_positions`, :func:`rotary_frequencies`).  Pairs are (p, p +
    all pairs) or, ``interleaved``, (2 p, 2 p + 1); values behind them are not
    turned.  Results are in ``dtype`` (default q's; float32 narrows to 16
    bits).  ``k`` may be None, and its result is.  ``out``: results to write
    into; they may be q and k."""
    yq, yk = out or (None, None)
    return _run(_binding.head_norm_rotary, q, stream, q, k, q_weight,
                k_weight, positions, frequencies, axes, interleaved, norm,
                eps, dtype, yq, yk)


def head_norm_rotary_backward(dq, dk, q, k=None, q_weight=None, k_weight=None,
                              positions=None, frequencies=None, axes=(),
                              interleaved=False, norm=True, eps=1e-6,
                              out=None, stream=None):
    """Gradients of q, k, q_weight and k_weight (fp32) of
    :func:`head_norm_rotary` (same arguments) for the gradients ``dq`` and
    ``dk`` of its results.  ``out``: tensors to write into (None for a
    weight's: not wanted); those of q and k may be dq and dk."""
    gq, gk, gqw, gkw = out or (None, None, None, None)
    return _run(_binding.head_norm_rotary_backward, q, stream, dq, dk, q, k,
                q_weight, k_weight, positions, frequencies, axes, interleaved,
                norm, eps, out is None, gq, gk, gqw, gkw)


def clip_gradients(grads, max_norm, out=None, norm=None, stream=None):
    """(clipped, norm): the norm of all values of ``grads`` (dense tensors)
    together and the tensors times min(1, max_norm / norm).  ``out``: tensors
    to write into, like ``grads`` (in place: ``grads`` itself); ``norm``: one
    fp32 value to write into (infinite past fp32's largest).  A value that is
    not finite leaves all as they are."""
    if not isinstance(grads, (list, tuple)):
        grads = list(grads)
    if not grads:
        raise ValueError("no gradients")
    in_place = out is grads
    norm, made = _run(_binding.clip_gradients, grads[0], stream, grads,
                      max_norm, None if in_place else out, in_place, norm)
    return (made if made is not None else out), norm
