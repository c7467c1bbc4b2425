"""The operators around a protected classifier, on torch tensors.

Group norm with an activation on channels-last maps (``group_norm``), 8-bit
matrices with a scale for each block of 128 (``fp8_quantize``) and their
product (``fp8_matmul``), and the scores of given classes or tokens
(``token_scores``), with the backward passes of the first and the last.
Checks of arguments, outputs and workspaces; the work runs in libctc.so's HIP
kernels (include/ctc.h states what each computes).

Every call takes tensors of one GPU, enqueues on ``stream`` (default: the
current stream of that GPU) and returns without waiting.  Outputs are
allocated unless given.  Tensors used on a stream that is not current have to
outlive their use there, as with any torch operator.  Wrong shapes, types or
devices raise ValueError before anything is enqueued; the library's own
refusals raise :class:`ctc.CtcError`.
"""

from __future__ import annotations

from functools import lru_cache
from typing import NamedTuple, Optional

import torch

from . import ctc

_REAL = {torch.float32: ctc.CTC_F32, torch.float16: ctc.CTC_F16,
         torch.bfloat16: ctc.CTC_BF16}
_BYTE = {torch.float8_e4m3fn: ctc.CTC_E4M3, torch.float8_e5m2: ctc.CTC_E5M2}
_QTYPE = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
_ACT = {"none": ctc.CTC_ACT_NONE, "relu": ctc.CTC_ACT_RELU,
        "silu": ctc.CTC_ACT_SILU}

BLOCK = 128

_current_raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _on(dev, stream):
    """(raw stream, whether it is dev's current one)."""
    if _current_raw is not None:
        cur = _current_raw(dev.index)
    else:
        cur = torch.cuda.current_stream(dev).cuda_stream
    if stream is None:
        return cur, True
    raw = stream if isinstance(stream, int) else stream.cuda_stream
    return raw, raw == cur


def _need(ok, msg, *args):
    if not ok:
        raise ValueError(msg % args if args else msg)


def _device(t, name):
    _need(isinstance(t, torch.Tensor) and t.is_cuda, "%s must be a GPU tensor",
          name)
    return t.device


def _like(t, name, dtype, shape, dev):
    """A contiguous tensor of that type, shape and device."""
    if t is None:
        return None
    _need(isinstance(t, torch.Tensor) and t.dtype == dtype
          and t.shape == shape and t.device == dev and t.is_contiguous(),
          "%s must be a contiguous %s tensor of shape %s on %s", name, dtype,
          tuple(shape), dev)
    return t.data_ptr()


def _rows(t, name, dev=None):
    """Row stride of a matrix whose rows are contiguous."""
    _need(isinstance(t, torch.Tensor) and t.dim() == 2 and
          (dev is None or t.device == dev), "%s must be a matrix%s", name,
          "" if dev is None else " on %s" % dev)
    _need(t.stride(1) == 1 or t.shape[1] <= 1,
          "the rows of %s must be contiguous", name)
    if t.shape[0] <= 1:
        # (torch keeps no meaningful stride for a single row)
        return max(t.shape[1], t.stride(0)) if t.shape[1] else 0
    _need(t.stride(0) >= t.shape[1], "the rows of %s overlap", name)
    return t.stride(0)


def _workspace(nbytes, dev, stream, current):
    """(tensor, address) of device scratch for one call."""
    if not nbytes:
        return None, None
    ws = torch.empty(nbytes, dtype=torch.uint8, device=dev)
    if not current:
        # allocated on the current stream, used on another
        if isinstance(stream, int):
            stream = torch.cuda.ExternalStream(stream, device=dev)
        ws.record_stream(stream)
    return ws, ws.data_ptr()


class _Device:
    """Makes dev current for the launch (nothing to do on one GPU)."""

    def __init__(self, dev):
        self.dev = dev
        self.prev = -1

    def __enter__(self):
        if torch.cuda.current_device() != self.dev.index:
            self.prev = torch.cuda.current_device()
            torch.cuda.set_device(self.dev)

    def __exit__(self, *exc):
        if self.prev >= 0:
            torch.cuda.set_device(self.prev)
        return False


# -------------------------------------------------------------- group norm

@lru_cache(maxsize=512)
def _norm_bytes(dtype, n, hw, c, groups, backward):
    return ctc.ctc_group_norm_workspace_bytes(dtype, n, hw, c, groups,
                                              backward)


def _map(x, groups, act):
    dev = _device(x, "x")
    _need(x.dtype in _REAL, "x must be float32, float16 or bfloat16")
    _need(x.dim() >= 2 and x.is_contiguous(),
          "x must be a contiguous [n, ..., c] map")
    _need(act in _ACT, "act must be one of %s", sorted(_ACT))
    n, c = x.shape[0], x.shape[-1]
    _need(groups >= 1 and c >= 1 and c % groups == 0,
          "%d groups do not divide %d channels", groups, c)
    hw = 1
    for d in x.shape[1:-1]:
        hw *= d
    _need(hw >= 1, "x has no pixels")
    return dev, n, hw, c


def group_norm(x, groups, gamma=None, beta=None, residual=None, act="none",
               carry=False, eps=1e-5, out=None, stream=None):
    """y, mean, rstd of a channels-last map ``x`` [n, ..., c]:
    ``y = act((x - mean) * rstd * gamma + beta (+ residual))`` with
    statistics over each image's pixels and each of ``groups`` channel groups
    (mean and rstd [n, groups], fp32).  ``act`` is "none", "relu" or "silu".
    With ``carry`` the last channel is a carry-through checksum, which takes
    no part and passes (plus the residual's).  ``out``: a (y, mean, rstd) of
    an earlier call to write into; its y may be x or residual."""
    dev, n, hw, c = _map(x, groups, act)
    if out is None:
        y = torch.empty_like(x)
        stats = torch.empty((2, n, groups), dtype=torch.float32, device=dev)
        mean, rstd = stats[0], stats[1]
    else:
        y, mean, rstd = out
    dt = _REAL[x.dtype]
    raw, current = _on(dev, stream)
    nb = _norm_bytes(dt, n, hw, c, groups, False)
    ws, wsp = _workspace(nb, dev, stream, current)
    with _Device(dev):
        ctc.ctc_group_norm_forward(
            dt, n, hw, c, groups, int(carry), x.data_ptr(),
            _like(gamma, "gamma", torch.float32, (c,), dev),
            _like(beta, "beta", torch.float32, (c,), dev),
            _like(residual, "residual", x.dtype, x.shape, dev), eps,
            _ACT[act], _like(y, "y", x.dtype, x.shape, dev),
            _like(mean, "mean", torch.float32, (n, groups), dev),
            _like(rstd, "rstd", torch.float32, (n, groups), dev), wsp, nb,
            raw)
    return y, mean, rstd


def group_norm_backward(dy, x, mean, rstd, groups, gamma=None, beta=None,
                        residual=None, act="none", carry=False, out=None,
                        stream=None):
    """dx, dresidual, dgamma, dbeta of :func:`group_norm` (same arguments,
    with the ``mean`` and ``rstd`` it returned); dresidual is None without a
    residual, dgamma and dbeta are always given (fp32).  ``out``: a tuple of
    an earlier call to write into, or of tensors and None (not wanted); its
    dx or its dresidual may be dy."""
    dev, n, hw, c = _map(x, groups, act)
    if out is None:
        dx = torch.empty_like(x)
        dr = None if residual is None else torch.empty_like(x)
        both = torch.empty((2, c), dtype=torch.float32, device=dev)
        dgamma, dbeta = both[0], both[1]
    else:
        dx, dr, dgamma, dbeta = out
    _need(dx is None or dr is None or n == 0
          or dx.data_ptr() != dr.data_ptr(), "dx and dresidual must differ")
    dt = _REAL[x.dtype]
    raw, current = _on(dev, stream)
    nb = _norm_bytes(dt, n, hw, c, groups, True)
    ws, wsp = _workspace(nb, dev, stream, current)
    f32 = torch.float32
    _need(dy is not None and mean is not None and rstd is not None,
          "dy, mean and rstd are needed")
    with _Device(dev):
        ctc.ctc_group_norm_backward(
            dt, n, hw, c, groups, int(carry),
            _like(dy, "dy", x.dtype, x.shape, dev), x.data_ptr(),
            _like(mean, "mean", f32, (n, groups), dev),
            _like(rstd, "rstd", f32, (n, groups), dev),
            _like(gamma, "gamma", f32, (c,), dev),
            _like(beta, "beta", f32, (c,), dev),
            _like(residual, "residual", x.dtype, x.shape, dev), _ACT[act],
            _like(dx, "dx", x.dtype, x.shape, dev),
            _like(dr, "dresidual", x.dtype, x.shape, dev),
            _like(dgamma, "dgamma", f32, (c,), dev),
            _like(dbeta, "dbeta", f32, (c,), dev), wsp, nb, raw)
    return dx, dr, dgamma, dbeta


# ---------------------------------------------------------- 8-bit matrices

def fp8_quantize(x, qtype="e4m3", block_rows=1, transpose=False, out=None,
                 stream=None):
    """(q, scales) of a matrix: ``x`` (or its transpose) in 8 bits with a
    scale for each ``block_rows`` (1 or 128) rows by 128 columns.  q is a
    float8 tensor whose rows begin at multiples of 16 bytes, scales
    [column blocks, row blocks] fp32; x is about q * scale."""
    dev = _device(x, "x")
    _need(x.dtype in _REAL, "x must be float32, float16 or bfloat16")
    _need(qtype in _QTYPE, "qtype must be one of %s", sorted(_QTYPE))
    _need(block_rows in (1, BLOCK), "block_rows must be 1 or %d", BLOCK)
    ldx = _rows(x, "x")
    rows, cols = x.shape
    qr, qc = (cols, rows) if transpose else (rows, cols)
    shape = (-(-qc // BLOCK), -(-qr // block_rows))
    if out is None:
        ld = -(-qc // 16) * 16
        q = torch.empty((qr, ld), dtype=_QTYPE[qtype], device=dev)
        if ld != qc:
            q = q[:, :qc]
        scales = torch.empty(shape, dtype=torch.float32, device=dev)
    else:
        q, scales = out
        _need(q.dtype == _QTYPE[qtype] and q.shape == (qr, qc),
              "q must be a %s matrix of shape %s", _QTYPE[qtype], (qr, qc))
    ldq = _rows_8bit(q, "q", dev)
    raw, _ = _on(dev, stream)
    with _Device(dev):
        ctc.ctc_fp8_quantize(
            _REAL[x.dtype], rows, cols, x.data_ptr(), ldx, _BYTE[q.dtype],
            block_rows, int(transpose), q.data_ptr(), ldq,
            _like(scales, "scales", torch.float32, shape, dev), shape[1],
            raw)
    return q, scales


def _rows_8bit(q, name, dev):
    """Row stride of an 8-bit matrix, all of whose rows can be read (and
    written) up to the next multiple of 16 columns."""
    ld = _rows(q, name, dev)
    rows, cols = q.shape
    wide = -(-cols // 16) * 16
    if rows == 0 or cols == 0:
        return wide
    if rows == 1:
        ld = wide
    _need(ld % 16 == 0 and q.data_ptr() % 16 == 0,
          "the rows of %s must begin at multiples of 16 bytes", name)
    _need((rows - 1) * ld + wide + q.storage_offset()
          <= q.untyped_storage().nbytes(),
          "the last row of %s must be allocated up to a multiple of 16 bytes",
          name)
    return ld


@lru_cache(maxsize=512)
def _matmul_bytes(ytype, m, n, k, b_block):
    return ctc.ctc_fp8_matmul_workspace_bytes(ytype, m, n, k, b_block)


def _scale_rows(scales, name, rows, kb, dev):
    """Rows to a scale (1 or 128) of a matrix's [kb, row blocks] scales."""
    _need(isinstance(scales, torch.Tensor) and scales.dtype == torch.float32
          and scales.dim() == 2 and scales.device == dev
          and scales.is_contiguous() and scales.shape[0] == kb
          and scales.shape[1] in (rows, -(-rows // BLOCK)),
          "%s must be a contiguous float32 tensor of shape (%d, %d) or "
          "(%d, %d) on %s", name, kb, rows, kb, -(-rows // BLOCK), dev)
    return 1 if scales.shape[1] == rows else BLOCK


def fp8_matmul(a, a_scales, b, b_scales, bias=None, act="none",
               dtype=torch.float16, out=None, stream=None):
    """act(A @ B.T + bias) in ``dtype`` for 8-bit matrices a [m, k] and
    b [n, k] with the scales of :func:`fp8_quantize` (A and B are the values
    they stand for)."""
    dev = _device(a, "a")
    _need(a.dtype in _BYTE and isinstance(b, torch.Tensor)
          and b.dtype in _BYTE, "a and b must be float8 tensors")
    lda, ldb = _rows_8bit(a, "a", dev), _rows_8bit(b, "b", dev)
    (m, k), n = a.shape, b.shape[0]
    _need(b.shape[1] == k, "a has %d columns, b %d", k, b.shape[1])
    _need(act in _ACT, "act must be one of %s", sorted(_ACT))
    kb = -(-k // BLOCK)
    ab = _scale_rows(a_scales, "a_scales", m, kb, dev)
    bb = _scale_rows(b_scales, "b_scales", n, kb, dev)
    if out is None:
        _need(dtype in _REAL, "dtype must be float32, float16 or bfloat16")
        out = torch.empty((m, n), dtype=dtype, device=dev)
    _need(out.dtype in _REAL and out.shape == (m, n),
          "out must be a real matrix of shape %s", (m, n))
    ldy = _rows(out, "out", dev)
    raw, current = _on(dev, stream)
    nb = _matmul_bytes(_REAL[out.dtype], m, n, k, bb)
    ws, wsp = _workspace(nb, dev, stream, current)
    with _Device(dev):
        ctc.ctc_fp8_matmul(
            _BYTE[a.dtype], _BYTE[b.dtype], _REAL[out.dtype], m, n, k,
            a.data_ptr(), lda, a_scales.data_ptr(), a_scales.shape[1], ab,
            b.data_ptr(), ldb, b_scales.data_ptr(), b_scales.shape[1], bb,
            _like(bias, "bias", torch.float32, (n,), dev), _ACT[act],
            out.data_ptr(), ldy, wsp, nb, raw)
    return out


# ------------------------------------------------------------------ scores

class TokenScores(NamedTuple):
    """Scores of rows of logits (fp32, int32): see :func:`token_scores`."""
    lse: torch.Tensor
    entropy: torch.Tensor
    logprob: Optional[torch.Tensor]
    rank: Optional[torch.Tensor]
    top_ids: Optional[torch.Tensor]
    top_logprobs: Optional[torch.Tensor]


@lru_cache(maxsize=512)
def _scores_bytes(rows, vocab, top_k):
    return ctc.ctc_token_scores_workspace_bytes(rows, vocab, top_k)


def _logits(logits):
    dev = _device(logits, "logits")
    _need(logits.dtype in _REAL,
          "logits must be float32, float16 or bfloat16")
    ld = _rows(logits, "logits")
    _need(logits.shape[1] >= 1, "logits without columns")
    return dev, logits.shape[0], logits.shape[1], ld


def token_scores(logits, targets=None, top_k=0, out=None, stream=None):
    """Scores of ``logits`` [rows, vocab] (rows may be strided: a protected
    classifier's ``out[:, :classes]``): log-sum-exp, entropy in nats, and for
    int32 ``targets`` [rows] (negative: none) the log probability and the
    rank, and the ``top_k`` best alternatives with their log probabilities
    (ties to the lower index; -1 and -inf where there is none).  ``out``: a
    TokenScores of an earlier call to write into."""
    dev, rows, vocab, ld = _logits(logits)
    f32, i32 = torch.float32, torch.int32
    given = targets is not None
    if out is None:
        f = torch.empty((3 if given else 2, rows), dtype=f32, device=dev)
        out = TokenScores(
            f[0], f[1], f[2] if given else None,
            torch.empty(rows, dtype=i32, device=dev) if given else None,
            torch.empty((rows, top_k), dtype=i32, device=dev) if top_k
            else None,
            torch.empty((rows, top_k), dtype=f32, device=dev) if top_k
            else None)
    raw, current = _on(dev, stream)
    nb = _scores_bytes(rows, vocab, top_k)
    ws, wsp = _workspace(nb, dev, stream, current)
    with _Device(dev):
        ctc.ctc_token_scores_forward(
            _REAL[logits.dtype], rows, vocab, logits.data_ptr(), ld,
            _like(targets, "targets", i32, (rows,), dev), top_k,
            _like(out.lse, "lse", f32, (rows,), dev),
            _like(out.logprob, "logprob", f32, (rows,), dev),
            _like(out.entropy, "entropy", f32, (rows,), dev),
            _like(out.rank, "rank", i32, (rows,), dev),
            _like(out.top_ids, "top_ids", i32, (rows, top_k), dev),
            _like(out.top_logprobs, "top_logprobs", f32, (rows, top_k), dev),
            wsp, nb, raw)
    return out


def token_scores_backward(logits, targets, lse, entropy=None, g_lse=None,
                          g_logprob=None, g_entropy=None, out=None,
                          stream=None):
    """Gradient of the scores' lse, logprob and entropy with respect to the
    logits, given those of the loss with respect to them (each [rows] fp32 or
    None).  ``out`` may be logits itself."""
    dev, rows, vocab, ld = _logits(logits)
    f32, shape = torch.float32, (rows,)
    if out is None:
        out = torch.empty((rows, vocab), dtype=logits.dtype, device=dev)
    _need(out.dtype == logits.dtype and out.shape == logits.shape,
          "out must be like logits")
    ldd = _rows(out, "out", dev)
    _need(lse is not None, "lse is needed")
    raw, _ = _on(dev, stream)
    with _Device(dev):
        ctc.ctc_token_scores_backward(
            _REAL[logits.dtype], rows, vocab, logits.data_ptr(), ld,
            _like(targets, "targets", torch.int32, shape, dev),
            _like(lse, "lse", f32, shape, dev),
            _like(entropy, "entropy", f32, shape, dev),
            _like(g_lse, "g_lse", f32, shape, dev),
            _like(g_logprob, "g_logprob", f32, shape, dev),
            _like(g_entropy, "g_entropy", f32, shape, dev), out.data_ptr(),
            ldd, raw)
    return out
