"""The operators of the output head's way to a token, on torch tensors: MXFP4 matrices (`mx4_quantize`, `mx4_dequantize`,
`mx4_matmul`) and rules on logits (`logits_rules`).  Marshalling only: each call checks its tensors, allocates its result with
torch and enqueues one kernel of libsdfp on the tensors' device and that device's current stream.  What the checks refuse
raises SdError (SD_EINVAL) before anything is enqueued.  Nothing is recorded for a gradient."""
from __future__ import annotations

import ctypes

import torch

from . import binding as B

# A call's time on the host is its cost wherever the kernel takes a few microseconds, so the checks below use the cheapest form
# of each question: device indexes instead of device objects, the raw handle of the current stream (torch.cuda.current_stream
# builds an object: 2.0 us against 0.1), exceptions for what is no tensor at all.
_CODES = {torch.float32: B.SD_F32, torch.bfloat16: B.SD_BF16}
_raw_stream = torch._C._cuda_getCurrentRawStream
_current_device = torch._C._cuda_getDevice       # (a tensor on a GPU exists: the runtime is up)
_END = 1 << 31                                    # sizes are 32-bit at the entry points, and ctypes would cut larger ones


def _refuse(what):
    raise B.SdError(B.SD_EINVAL, what)


def _call(name, index, *args):
    """The entry point `name` with (*args, current stream of device `index`), with the device current; a code other than SD_OK
    is raised."""
    fn = getattr(B.load_library(), name)
    if _current_device() == index:
        rc = fn(*args, _raw_stream(index))
    else:
        with torch.cuda.device(index):
            rc = fn(*args, _raw_stream(index))
    if rc != B.SD_OK:
        raise B.SdError(rc, name)


def _rows(t, where):
    """(rows, columns, distance of rows, type code, device index) of a 2-D tensor on a GPU whose rows are contiguous."""
    try:
        n, c = t.shape
        ld, step = t.stride()
        code, index = _CODES[t.dtype], t.get_device()
    except (AttributeError, ValueError, KeyError, RuntimeError, TypeError):   # no tensor, not two dimensions, another type
        _refuse(where)
    if n == 1:
        ld = c
    if index < 0 or not 0 < n < _END or not 0 < c < _END or (step != 1 and c != 1) or ld < c:
        _refuse(where)
    return n, c, ld, code, index


def _array(t, dtypes, shape, index, where):
    """The address of a contiguous tensor of one of `dtypes` and of `shape` (None: any vector) on device `index`."""
    try:
        if t.dtype in dtypes and t.get_device() == index and t.is_contiguous() and (t.shape == shape if shape is not None else t.dim() == 1):
            return t.data_ptr()
    except AttributeError:      # no tensor at all
        pass
    _refuse(where)


_I32, _I64, _F32, _BITS = (torch.int32,), (torch.int64,), (torch.float32,), (torch.int32, torch.uint32)


class Mx4:
    """A matrix of rows x cols in MXFP4: its panels, a uint8 tensor of sd_mx4_bytes(rows, cols) bytes (include/sdfp.h)."""

    __slots__ = ("data", "rows", "cols")

    def __init__(self, data, rows, cols):
        try:
            ok = (data.dtype is torch.uint8 and data.is_cuda and data.is_contiguous() and 0 < rows < _END and 0 < cols < _END and
                  data.numel() >= (rows + 63) // 64 * ((cols + 127) // 128) * 4352 and data.data_ptr() % 256 == 0)
        except (AttributeError, TypeError):
            ok = False
        if not ok:
            _refuse("Mx4: a contiguous, 256-byte aligned uint8 tensor of at least the matrix's size on a GPU")
        self.data, self.rows, self.cols = data, rows, cols

    def __repr__(self):
        return f"Mx4({self.rows} x {self.cols}, {self.data.device})"


def mx4_quantize(x) -> Mx4:
    """Rows of float32 or bfloat16 in MXFP4 (sd_mx4_quantize)."""
    rows, cols, ld, code, index = _rows(x, "mx4_quantize: x")
    n = (rows + 63) // 64 * ((cols + 127) // 128) * 4352
    data = x.new_empty(n, dtype=torch.uint8)
    _call("sd_mx4_quantize", index, x.data_ptr(), code, ld, rows, cols, data.data_ptr(), n)
    q = Mx4.__new__(Mx4)
    q.data, q.rows, q.cols = data, rows, cols
    return q


def mx4_dequantize(q: Mx4, dtype=torch.float32):
    """The values of an MXFP4 matrix as rows of float32 or bfloat16, both exact (sd_mx4_dequantize)."""
    code = _CODES.get(dtype)
    if not isinstance(q, Mx4) or code is None:
        _refuse("mx4_dequantize: q, dtype")
    d, cols = q.data, q.cols
    x = d.new_empty((q.rows, cols), dtype=dtype)
    _call("sd_mx4_dequantize", d.get_device(), d.data_ptr(), d.numel(), q.rows, cols, x.data_ptr(), code, cols)
    return x


def mx4_matmul(x, w: Mx4, gain=None, eps: float = 1e-5, out_dtype=None):
    """x w^T (sd_mx4_matmul).  x: rows of float32 or bfloat16, or an Mx4; gain (float32 x only): RMS-normalise the rows and
    multiply by it first.  The result has x's type, float32 for an Mx4, or out_dtype (float32 or bfloat16)."""
    if not isinstance(w, Mx4):
        _refuse("mx4_matmul: w")
    wd, n = w.data, w.rows
    index = wd.get_device()
    if isinstance(x, Mx4):
        m, k, xd, code, dtype = x.rows, x.cols, x.data, B.SD_MX4, torch.float32
        ld, on = xd.numel(), xd.get_device()
    else:
        m, k, ld, code, on = _rows(x, "mx4_matmul: x")
        xd, dtype = x, x.dtype
    if k != w.cols or on != index:
        _refuse("mx4_matmul: x and w of one width on one device")
    if out_dtype is not None:
        dtype = out_dtype
    y_code = _CODES.get(dtype)
    if y_code is None or (gain is not None and code != B.SD_F32):
        _refuse("mx4_matmul: out_dtype, or a gain without float32 x")
    g = None if gain is None else _array(gain, _F32, (k,), index, "mx4_matmul: gain")
    y = xd.new_empty((m, n)) if dtype is xd.dtype else wd.new_empty((m, n), dtype=dtype)
    _call("sd_mx4_matmul", index, wd.data_ptr(), wd.numel(), n, k, xd.data_ptr(), code, ld, m, g, eps, y.data_ptr(), y_code, n)
    return y


def logits_rules(logits, tokens=None, begin=None, end=None, *, repetition: float = 1.0, presence: float = 0.0, frequency: float = 0.0,
                 bias=None, allowed=None, mask_row=None, out=None):
    """Rows of logits [rows][vocab] (float32 or bfloat16) under penalties, bias and masks (sd_logits_rules).

    tokens (int32), begin and end (int64 [rows]): row i's history is tokens[begin[i]:end[i]]; needed if a penalty is set.
    bias: float32 [vocab].  allowed: int32 or uint32 [n_masks][ceil(vocab / 32)], bit j % 32 of word j // 32 allows token j;
    mask_row: int32 [rows], the mask of each row (-1: none); by default row i has mask i, or all have the only one.
    out: where the result goes (`logits` itself: in place); by default a new tensor."""
    rows, vocab, ld, code, index = _rows(logits, "logits_rules: logits")
    if out is None:
        out, ld_out = torch.empty_like(logits) if ld == vocab else logits.new_empty((rows, vocab)), vocab
    else:
        r, v, ld_out, c, on = _rows(out, "logits_rules: out")
        if r != rows or v != vocab or c != code or on != index:
            _refuse("logits_rules: out")
    t = b = e = p_bias = p_allowed = m = None
    n = n_masks = 0
    if repetition != 1.0 or presence != 0.0 or frequency != 0.0:
        t, n = _array(tokens, _I32, None, index, "logits_rules: tokens"), tokens.numel()
        b = _array(begin, _I64, (rows,), index, "logits_rules: begin")
        e = _array(end, _I64, (rows,), index, "logits_rules: end")
    if bias is not None:
        p_bias = _array(bias, _F32, (vocab,), index, "logits_rules: bias")
    if allowed is not None:
        n_masks = allowed.shape[0] if isinstance(allowed, torch.Tensor) and allowed.dim() else 0
        if not 0 < n_masks < _END:
            _refuse("logits_rules: allowed")
        p_allowed = _array(allowed, _BITS, (n_masks, (vocab + 31) // 32), index, "logits_rules: allowed")
        if mask_row is not None:
            m = _array(mask_row, _I32, (rows,), index, "logits_rules: mask_row")
    _call("sd_logits_rules", index, logits.data_ptr(), code, ld, rows, vocab,
          ctypes.byref(B.SdRules(repetition, presence, frequency, p_bias, p_allowed, n_masks)), t, n, b, e, m, out.data_ptr(), ld_out)
    return out
