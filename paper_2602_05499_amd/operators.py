"""The operators of the output head's way to a token, on torch tensors: MXFP4 matrices (`mx4_quantize`, `mx4_dequantize`,
`mx4_matmul`) and rules on logits (`logits_rules`).  Marshalling only: each call checks its tensors, allocates its result with
torch and enqueues one kernel of libsdfp on the tensors' device and that device's current stream.  What the checks refuse
raises SdError (SD_EINVAL) before anything is enqueued."""
from __future__ import annotations

import torch

from . import binding as B

_CODES = {torch.float32: B.SD_F32, torch.bfloat16: B.SD_BF16}


def _require(ok, what):
    if not ok:
        raise B.SdError(B.SD_EINVAL, what)


def _check(rc, where):
    if rc != B.SD_OK:
        raise B.SdError(rc, where)


def _on(device, fn, *args):
    """fn(*args, current stream of device), with the device current."""
    if torch.cuda.current_device() == device.index:
        return fn(*args, torch.cuda.current_stream(device).cuda_stream)
    with torch.cuda.device(device):
        return fn(*args, torch.cuda.current_stream(device).cuda_stream)


def _rows(t, where, types=_CODES):
    """(rows, columns, distance of rows) of a 2-D tensor whose rows are contiguous."""
    _require(isinstance(t, torch.Tensor) and t.is_cuda and t.dim() == 2 and t.dtype in types, where)
    n, c = t.shape
    _require(n > 0 and c > 0 and (c == 1 or t.stride(1) == 1), where)
    ld = t.stride(0) if n > 1 else c
    _require(ld >= c, where)
    return n, c, ld


def _vector(t, dtype, n, device, where):
    _require(isinstance(t, torch.Tensor) and t.device == device and t.dtype == dtype and t.dim() == 1 and t.is_contiguous() and
             (n is None or t.numel() == n), where)
    return t.data_ptr()


class Mx4:
    """A matrix of rows x cols in MXFP4: its panels, a uint8 tensor of sd_mx4_bytes(rows, cols) bytes (include/sdfp.h)."""

    __slots__ = ("data", "rows", "cols")

    def __init__(self, data, rows, cols):
        need = B.sd_mx4_bytes(rows, cols)
        _require(isinstance(data, torch.Tensor) and data.is_cuda and data.dtype == torch.uint8 and data.is_contiguous() and
                 need > 0 and data.numel() >= need and data.data_ptr() % 256 == 0, "Mx4: a contiguous, aligned uint8 tensor of the matrix's size")
        self.data, self.rows, self.cols = data, rows, cols

    def __repr__(self):
        return f"Mx4({self.rows} x {self.cols}, {self.data.device})"


def mx4_quantize(x) -> Mx4:
    """Rows of float32 or bfloat16 in MXFP4 (sd_mx4_quantize)."""
    rows, cols, ld = _rows(x, "mx4_quantize: x")
    n = B.sd_mx4_bytes(rows, cols)
    q = torch.empty(n, dtype=torch.uint8, device=x.device)
    _check(_on(x.device, B.sd_mx4_quantize, x.data_ptr(), _CODES[x.dtype], ld, rows, cols, q.data_ptr(), n), "sd_mx4_quantize")
    return Mx4(q, rows, cols)


def mx4_dequantize(q: Mx4, dtype=torch.float32):
    """The values of an MXFP4 matrix as rows of float32 or bfloat16, both exact (sd_mx4_dequantize)."""
    _require(isinstance(q, Mx4) and dtype in _CODES, "mx4_dequantize: q, dtype")
    x = torch.empty(q.rows, q.cols, dtype=dtype, device=q.data.device)
    _check(_on(x.device, B.sd_mx4_dequantize, q.data.data_ptr(), q.data.numel(), q.rows, q.cols, x.data_ptr(), _CODES[dtype], q.cols),
           "sd_mx4_dequantize")
    return x


def mx4_matmul(x, w: Mx4, gain=None, eps: float = 1e-5, out_dtype=None):
    """x w^T (sd_mx4_matmul).  x: rows of float32 or bfloat16, or an Mx4; gain (float32 x only): RMS-normalise the rows and
    multiply by it first.  The result has x's type, float32 for an Mx4, or out_dtype (float32 or bfloat16)."""
    _require(isinstance(w, Mx4), "mx4_matmul: w")
    dev = w.data.device
    if isinstance(x, Mx4):
        m, k, ldx, code, ptr, dt = x.rows, x.cols, x.data.numel(), B.SD_MX4, x.data.data_ptr(), torch.float32
        _require(x.data.device == dev, "mx4_matmul: x and w on one device")
    else:
        m, k, ldx = _rows(x, "mx4_matmul: x")
        code, ptr, dt = _CODES[x.dtype], x.data_ptr(), x.dtype
        _require(x.device == dev, "mx4_matmul: x and w on one device")
    _require(k == w.cols, "mx4_matmul: columns of x and w")
    if out_dtype is not None:
        _require(out_dtype in _CODES, "mx4_matmul: out_dtype")
        dt = out_dtype
    g = None
    if gain is not None:
        _require(code == B.SD_F32, "mx4_matmul: a gain goes with float32 x")
        g = _vector(gain, torch.float32, k, dev, "mx4_matmul: gain")
    y = torch.empty(m, w.rows, dtype=dt, device=dev)
    _check(_on(dev, B.sd_mx4_matmul, w.data.data_ptr(), w.data.numel(), w.rows, k, ptr, code, ldx, m, g, eps, y.data_ptr(),
               _CODES[dt], w.rows), "sd_mx4_matmul")
    return y


def logits_rules(logits, tokens=None, begin=None, end=None, *, repetition: float = 1.0, presence: float = 0.0, frequency: float = 0.0,
                 bias=None, allowed=None, mask_row=None, out=None):
    """Rows of logits [rows][vocab] (float32 or bfloat16) under penalties, bias and masks (sd_logits_rules).

    tokens (int32), begin and end (int64 [rows]): row i's history is tokens[begin[i]:end[i]]; needed if a penalty is set.
    bias: float32 [vocab].  allowed: int32 or uint32 [n_masks][ceil(vocab / 32)], bit j % 32 of word j // 32 allows token j;
    mask_row: int32 [rows], the mask of each row (-1: none); by default row i has mask i, or all have the only one.
    out: where the result goes (`logits` itself: in place); by default a new tensor."""
    rows, vocab, ld = _rows(logits, "logits_rules: logits")
    dev = logits.device
    if out is None:
        out = torch.empty(rows, vocab, dtype=logits.dtype, device=dev)
        ld_out = vocab
    else:
        r, v, ld_out = _rows(out, "logits_rules: out", (logits.dtype,))
        _require((r, v) == (rows, vocab) and out.device == dev, "logits_rules: out")
    t = b = e = m = None
    n = 0
    if repetition != 1.0 or presence != 0.0 or frequency != 0.0:
        t, n = _vector(tokens, torch.int32, None, dev, "logits_rules: tokens"), tokens.numel()
        b = _vector(begin, torch.int64, rows, dev, "logits_rules: begin")
        e = _vector(end, torch.int64, rows, dev, "logits_rules: end")
    rules = B.SdRules(repetition, presence, frequency, None, None, 0)
    if bias is not None:
        rules.bias = _vector(bias, torch.float32, vocab, dev, "logits_rules: bias")
    if allowed is not None:
        _require(isinstance(allowed, torch.Tensor) and allowed.device == dev and allowed.dtype in (torch.int32, torch.uint32) and
                 allowed.dim() == 2 and allowed.is_contiguous() and allowed.shape[0] > 0 and allowed.shape[1] == (vocab + 31) // 32,
                 "logits_rules: allowed")
        rules.allowed, rules.n_masks = allowed.data_ptr(), allowed.shape[0]
        if mask_row is not None:
            m = _vector(mask_row, torch.int32, rows, dev, "logits_rules: mask_row")
    _check(_on(dev, B.sd_logits_rules, logits.data_ptr(), _CODES[logits.dtype], ld, rows, vocab, rules, t, n, b, e, m, out.data_ptr(),
               ld_out), "sd_logits_rules")
    return out
