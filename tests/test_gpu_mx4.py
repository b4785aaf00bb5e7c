"""MXFP4 quantisation, reading back and product against plain implementations in 64 bits, at the sizes and values where they
can go wrong: one row and column, ragged panels, strided and unaligned rows, ties, denormals, infinities and NaN."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


@pytest.fixture(scope="module")
def P():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2602_05499_amd as P
    return P


def quantize64(x):
    """(codes [rows][cols], scale bytes [rows][blocks]) of a float array, by the definition in float64."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    nb = -(-cols // 32)
    xp = np.zeros((rows, nb * 32))
    xp[:, :cols] = x
    xb = xp.reshape(rows, nb, 32)
    finite = np.isfinite(xb).all(-1)
    amax = np.where(finite, np.abs(np.where(np.isfinite(xb), xb, 0.0)).max(-1), 0.0)
    e = np.where(amax > 0, np.maximum(np.frexp(amax)[1] - 1 - 2, -126), -126)
    a = np.abs(np.where(finite[..., None], xb, 0.0)) / np.exp2(e.astype(np.float64))[..., None]
    code = np.zeros(a.shape, np.int64)
    for i in range(7):
        mid = (GRID[i] + GRID[i + 1]) / 2
        code += (a > mid) | ((a == mid) & (i % 2 == 1))
    code += 8 * np.signbit(xb) * finite[..., None]
    return code.reshape(rows, -1)[:, :cols], np.where(finite, e + 127, 255).astype(np.int64)


def values64(code, e):
    """float64 values of codes and scale bytes."""
    s = np.where(e == 255, np.nan, np.exp2(np.minimum(e, 254) - 127.0))
    v = GRID[code & 7] * np.where(code & 8, -1.0, 1.0)
    return v * np.repeat(s, 32, axis=1)[:, :code.shape[1]]


def panels(code, e):
    """The bytes of the panel format, element by element as the header states it."""
    rows, cols = code.shape
    rp, cp = -(-rows // 64), -(-cols // 128)
    q = np.zeros((rp, cp, 4352), np.uint8)
    for r in range(rows):
        t, rr = r % 64 // 16, r % 16
        for c in range(cols):
            b, i = c % 128 // 32, c % 32
            q[r // 64, c // 128, ((t * 4 + b) * 16 + rr) * 16 + i // 2] |= code[r, c] << (4 * (i % 2))
        for blk in range(e.shape[1]):
            q[r // 64, blk // 4, 4096 + (blk % 4 * 16 + rr) * 4 + t] = e[r, blk]
    return q.reshape(-1)


def _rows(rows, cols, dtype, seed):
    import torch
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, cols)) * np.exp2(rng.integers(-6, 7, (rows, 1)).astype(float))
    return torch.from_numpy(x.astype(np.float32)).to(dtype).cuda()


def _np(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 20), (5, 1000), (64, 128), (65, 129), (16, 31), (130, 257), (3, 4096), (200, 33)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_quantize_and_read_back(P, rows, cols, dtype):
    import torch
    dt = getattr(torch, dtype)
    x = _rows(rows, cols, dt, rows * 7 + cols)
    q = P.mx4_quantize(x)
    code, e = quantize64(_np(x))
    got = q.data.cpu().numpy()
    want = panels(code, e)
    kp = -(-cols // 128)
    g, w = got.reshape(-1, kp, 4352), want.reshape(-1, kp, 4352)
    assert np.array_equal(g[..., :4096], w[..., :4096])
    pad = np.ones(w[..., 4096:].shape, bool)       # scale bytes of blocks past the matrix are not pinned
    pad[w[..., 4096:] > 0] = False
    assert np.array_equal(np.where(pad, 0, g[..., 4096:]), w[..., 4096:])
    for out in (torch.float32, torch.bfloat16):
        back = P.mx4_dequantize(q, out)
        assert back.dtype == out and np.array_equal(_np(back), values64(code, e))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_quantize_edges(P, dtype):
    """Zeros, negative zeros, denormals, the largest and smallest magnitudes, every tie, blocks with infinities and NaN."""
    import torch
    dt = getattr(torch, dtype)
    top = float(torch.finfo(dt).max)
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0])
    blocks = [np.zeros(32), -np.zeros(32), np.full(32, 2.0 ** -126), np.full(32, 2.0 ** -133), np.r_[2.0 ** -125, np.full(31, -2.0 ** -127)],
              np.r_[top, np.full(31, -1e30)], np.r_[np.inf, np.ones(31)], np.r_[np.ones(31), -np.inf], np.r_[np.ones(5), np.nan, np.ones(26)]]
    for s in (-60, 0, 60):
        blocks.append(np.r_[4.0, ties, -ties, np.nextafter(np.float32(2.5), np.float32(3)).astype(float), np.zeros(14)] * 2.0 ** s)
    x = torch.tensor(np.stack(blocks).reshape(2, -1)).to(dt)
    code, e = quantize64(x.double().numpy())
    q = P.mx4_quantize(x.cuda())
    assert np.array_equal(_np(P.mx4_dequantize(q)), values64(code, e), equal_nan=True)
    v = _np(P.mx4_dequantize(q, torch.bfloat16))
    assert np.array_equal(v, values64(code, e), equal_nan=True)
    assert np.isnan(v).sum() == 3 * 32 and np.array_equal(np.signbit(v[0, 32:64]), np.ones(32, bool))


def test_strided_and_unaligned_rows(P):
    import torch
    for dt in (torch.float32, torch.bfloat16):
        big = _rows(90, 301, dt, 5)
        for view in (big[3:75, 1:222], big[::2, 3:], big[:, 300:]):
            code, e = quantize64(_np(view))
            assert np.array_equal(_np(P.mx4_dequantize(P.mx4_quantize(view))), values64(code, e))
            w = P.mx4_quantize(_rows(70, view.shape[1], torch.float32, 6))
            a, b = P.mx4_matmul(view, w), P.mx4_matmul(view.contiguous(), w)
            assert torch.equal(a, b)


def _tolerance(x, w, k, out):
    """|error| allowed per output: each of the at most 3 ceil(k / 32) + 16 additions of the chain that sums the products rounds
    (or truncates) by at most 2^-23 of a partial sum, which sum |x w| bounds; the result's own rounding on top."""
    import torch
    s = np.abs(x) @ np.abs(w).T
    y = np.abs(x @ w.T)
    return (3 * -(-k // 32) + 16) * 2.0 ** -23 * s + (2.0 ** -8 * y if out == torch.bfloat16 else 0.0) + 1e-37


SIZES = [(1, 1, 1), (1, 64, 128), (2, 65, 129), (1, 1000, 4096), (3, 130, 777), (4, 64, 20), (5, 300, 1025), (16, 129, 640), (17, 70, 300),
         (37, 1003, 777), (33, 64, 2048), (64, 200, 512), (100, 77, 96), (300, 520, 400), (257, 1100, 1280), (513, 640, 257)]


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("kind", ["float32", "bfloat16", "mx4"])
def test_matmul(P, m, n, k, kind):
    import torch
    wf = _rows(n, k, torch.float32, m + n + k)
    wq = P.mx4_quantize(wf)
    wv = values64(*quantize64(_np(wf)))
    if kind == "mx4":
        xf = _rows(m, k, torch.float32, m * 3 + n)
        x, xv = P.mx4_quantize(xf), values64(*quantize64(_np(xf)))
    else:
        x = _rows(m, k, getattr(torch, kind), m * 3 + n)
        xv = _np(x)
    for out in (torch.float32, torch.bfloat16):
        y = P.mx4_matmul(x, wq, out_dtype=out)
        assert y.shape == (m, n) and y.dtype == out
        assert (np.abs(_np(y) - xv @ wv.T) <= _tolerance(xv, wv, k, out)).all()
        assert torch.equal(y, P.mx4_matmul(x, wq, out_dtype=out))
    assert P.mx4_matmul(x, wq).dtype == (torch.bfloat16 if kind == "bfloat16" else torch.float32)


@pytest.mark.parametrize("m,n,k", [(1, 100, 4096), (1, 65, 33), (3, 70, 1000), (9, 64, 513), (16, 64, 128), (40, 200, 640), (300, 300, 300)])
def test_matmul_with_gain(P, m, n, k):
    """RMS-normalised rows: the factor's own error is a few roundings and that of a sum of k squares (at most
    (ceil(k / 32) + 16) 2^-23 relative), the multiplication by the gain rounds once."""
    import torch
    x, wf = _rows(m, k, torch.float32, 1), _rows(n, k, torch.float32, 2)
    gain = 1.0 + 0.3 * _rows(1, k, torch.float32, 3)[0].clamp(-2, 2)
    wv = values64(*quantize64(_np(wf)))
    xv = _np(x)
    xh = xv * _np(gain) / np.sqrt((xv ** 2).mean(-1, keepdims=True) + 1e-5)
    y = _np(P.mx4_matmul(x, P.mx4_quantize(wf), gain=gain, eps=1e-5))
    s = np.abs(xh) @ np.abs(wv).T
    tol = _tolerance(xh, wv, k, torch.float32) + (k / 32 + 24) * 2.0 ** -23 * s
    assert (np.abs(y - xh @ wv.T) <= tol).all()


@pytest.mark.parametrize("m", [1, 3, 16, 40, 300])
def test_infinities_and_nan(P, m):
    """A NaN block of w makes its output column NaN, one of x its row; infinite x follows IEEE arithmetic; nothing else changes.
    Large and tiny values stay finite."""
    import torch
    n, k = 70, 300
    wf = _rows(n, k, torch.float32, 8)
    wf[5, 40] = float("inf")
    wq, wv = P.mx4_quantize(wf), values64(*quantize64(_np(wf)))
    for dt in (torch.float32, torch.bfloat16):
        x = _rows(m, k, dt, 9)
        x[m // 2, 7] = float("inf")
        x[0, 299] = float("nan") if m > 1 else x[0, 299]
        y = _np(P.mx4_matmul(x, wq, out_dtype=torch.float32))
        xv = _np(x)
        with np.errstate(invalid="ignore"):
            want = np.stack([(xv[i] * wv).sum(-1) for i in range(m)])
        assert np.array_equal(np.isnan(y), np.isnan(want)) and np.isnan(want[:, 5]).all()
        assert np.array_equal(np.isinf(y), np.isinf(want)) and np.isinf(want).any()
        assert np.array_equal(y[np.isinf(y)], want[np.isinf(want)])
    xf = _rows(m, k, torch.float32, 10)
    xf[m - 1, 250] = float("nan")
    y = _np(P.mx4_matmul(P.mx4_quantize(xf), wq))
    bad = np.zeros((m, n), bool)
    bad[m - 1], bad[:, 5] = True, True
    assert np.array_equal(np.isnan(y), bad)
    big = torch.full((m, 32), 3.3e38, device="cuda")
    one = torch.zeros(2, 32, device="cuda")
    one[0, 3], one[1, 4] = 1.0, -1.0
    y = P.mx4_matmul(big, P.mx4_quantize(one))
    assert torch.equal(y, big[:, :2] * torch.tensor([1.0, -1.0], device="cuda"))


# rows and outputs that take each of the kernels for many rows, with ragged last tiles in both directions
TILES = {"float32": [(129, 11009), (300, 11009), (520, 11009)], "bfloat16": [(100, 6001), (200, 11009), (520, 11009)],
         "mx4": [(100, 8003), (1100, 7777)]}


@pytest.mark.parametrize("k", [20, 128, 130, 385, 512, 1000, 1281])
@pytest.mark.parametrize("kind,m,n", [(t, *mn) for t, v in TILES.items() for mn in v])
def test_matmul_of_many_rows(P, kind, m, n, k):
    """Every tile kernel at reduction lengths around its steps of 128, 256 and 512 columns; float32 with and without a gain; the
    plain products in float64 on the GPU."""
    import torch
    wq = P.mx4_quantize(_rows(n, k, torch.float32, k))
    wv = P.mx4_dequantize(wq).double()
    xf = _rows(m, k, torch.float32, k + 1)
    if kind == "mx4":
        x = P.mx4_quantize(xf)
        xv = P.mx4_dequantize(x).double()
    else:
        x = xf.to(getattr(torch, kind))
        xv = x.double()
    roundings = (3 * -(-k // 32) + 16) * 2.0 ** -23
    y = P.mx4_matmul(x, wq)
    tol = roundings * (xv.abs() @ wv.abs().t()) + (2.0 ** -8 * (xv @ wv.t()).abs() if kind == "bfloat16" else 0.0) + 1e-37
    assert ((y.double() - xv @ wv.t()).abs() <= tol).all()
    assert torch.equal(y, P.mx4_matmul(x, wq))
    if kind == "float32":
        gain = 1.0 + 0.3 * _rows(1, k, torch.float32, 3)[0].clamp(-2, 2)
        xh = xv * gain.double() / torch.sqrt((xv ** 2).mean(-1, keepdim=True) + 1e-5)
        y = P.mx4_matmul(x, wq, gain=gain, eps=1e-5)
        tol = (roundings + (k / 32 + 24) * 2.0 ** -23) * (xh.abs() @ wv.abs().t()) + 1e-37
        assert ((y.double() - xh @ wv.t()).abs() <= tol).all()


@pytest.mark.parametrize("kind,m,n", [(t, *mn) for t, v in TILES.items() for mn in v])
def test_nan_blocks_and_strides_of_many_rows(P, kind, m, n):
    """A NaN block of w, or of x, fills its output column or row and nothing else; x's rows may lie apart and unaligned, and what
    lies between and behind the rows of y is not touched."""
    import torch
    from paper_2602_05499_amd import binding as B
    k = 700
    wf = _rows(n, k, torch.float32, 8)
    wf[n - 2, 699] = float("nan")
    wf[70, 0] = float("inf")
    wq = P.mx4_quantize(wf)
    big = _rows(m, k + 5, torch.float32, 9)
    if kind == "mx4":
        big[m - 1, 300] = float("nan")
        x = P.mx4_quantize(big[:, 3:k + 3])
    else:
        x = big.to(getattr(torch, kind))[:, 3:k + 3]
    y = P.mx4_matmul(x, wq, out_dtype=torch.float32)
    bad = torch.zeros(m, n, dtype=torch.bool, device="cuda")
    bad[:, n - 2] = bad[:, 70] = True
    if kind == "mx4":
        bad[m - 1] = True
    else:
        assert torch.equal(P.mx4_matmul(x.contiguous(), wq, out_dtype=torch.float32).nan_to_num(), y.nan_to_num())
    assert torch.equal(torch.isnan(y), bad) and not torch.isinf(y).any()
    out = torch.full((m + 1, n + 3), 7.5, device="cuda")
    code, ptr, ld = (B.SD_MX4, x.data.data_ptr(), x.data.numel()) if kind == "mx4" else \
        ({"float32": B.SD_F32, "bfloat16": B.SD_BF16}[kind], x.data_ptr(), k + 5)
    assert B.sd_mx4_matmul(wq.data.data_ptr(), wq.data.numel(), n, k, ptr, code, ld, m, None, 0.0, out.data_ptr(), B.SD_F32, n + 3,
                           torch.cuda.current_stream().cuda_stream) == B.SD_OK
    assert torch.equal(out[:m, :n].nan_to_num(), y.nan_to_num()) and (out[m:] == 7.5).all() and (out[:, n:] == 7.5).all()


@pytest.mark.parametrize("m,n", [(4200, 8195), (1040, 1037)])
@pytest.mark.parametrize("kind", ["float32", "bfloat16", "mx4"])
def test_results_of_both_types_within_wider_rows(P, kind, m, n):
    """Results larger and smaller than the caches in both types, as rows at an odd distance, ending inside a panel: the values, and
    nothing beside them."""
    import torch
    from paper_2602_05499_amd import binding as B
    k = 130
    wq = P.mx4_quantize(_rows(n, k, torch.float32, 8))
    xf = _rows(m, k, torch.float32, 9)
    x = P.mx4_quantize(xf) if kind == "mx4" else xf.to(getattr(torch, kind))
    xv, wv = (P.mx4_dequantize(x) if kind == "mx4" else x).double(), P.mx4_dequantize(wq).double()
    want, mag = xv @ wv.t(), xv.abs() @ wv.abs().t()
    code, ptr, ld = (B.SD_MX4, x.data.data_ptr(), x.data.numel()) if kind == "mx4" else \
        ({"float32": B.SD_F32, "bfloat16": B.SD_BF16}[kind], x.data_ptr(), k)
    for out, y_code, step in ((torch.float32, B.SD_F32, 0.0), (torch.bfloat16, B.SD_BF16, 2.0 ** -8)):
        y = torch.full((m + 1, n + 6), 7.5, dtype=out, device="cuda")
        assert B.sd_mx4_matmul(wq.data.data_ptr(), wq.data.numel(), n, k, ptr, code, ld, m, None, 0.0, y[:, 3:].data_ptr(), y_code, n + 6,
                               torch.cuda.current_stream().cuda_stream) == B.SD_OK
        tol = (3 * -(-k // 32) + 16) * 2.0 ** -23 * mag + step * want.abs() + 1e-37
        assert ((y[:m, 3:n + 3].double() - want).abs() <= tol).all()
        assert (y[m:] == 7.5).all() and (y[:, :3] == 7.5).all() and (y[:, n + 3:] == 7.5).all()


@pytest.mark.parametrize("m", [1, 5, 16, 300])
@pytest.mark.parametrize("e", [0, 1, 2, 127, 250])
def test_scale_bytes_from_elsewhere(P, m, e):
    """Panels that the caller filled: every scale byte stands for 2^(e - 127), the smallest ones too, and the codes for their
    columns, low bits first.  Powers of two: the products are exact."""
    import torch
    n = 6400
    data = torch.zeros(P.sd_mx4_bytes(n, 128), dtype=torch.uint8, device="cuda").view(n // 64, 4352)
    data[:, 0] = 0x21                                   # row 0 of a panel: 0.5 and 1 in columns 0 and 1
    data[:, 4096] = e
    w = P.Mx4(data.reshape(-1), n, 128)
    v = P.mx4_dequantize(w)
    assert (v[0::64, 0] == 0.5 * 2.0 ** (e - 127)).all() and (v[0::64, 1] == 2.0 ** (e - 127)).all() and not v[:, 2:].any()
    f = 2.0 ** min(100, 250 - e)
    for col in (0, 1):
        want = torch.zeros(m, n, device="cuda")
        want[:, 0::64] = (0.5, 1.0)[col] * 2.0 ** (e - 127) * f
        x = torch.zeros(m, 128, device="cuda")
        x[:, col] = f
        for xs in (x, x.bfloat16(), P.mx4_quantize(x)):
            assert torch.equal(P.mx4_matmul(xs, w, out_dtype=torch.float32), want)


def test_first_calls_inside_a_capture(P):
    """Kernels of many rows captured, and replayed on other contents."""
    import torch
    w = P.mx4_quantize(_rows(11009, 300, torch.float32, 1))
    xs = [_rows(520, 300, torch.float32, 2), _rows(520, 300, torch.bfloat16, 3), P.mx4_quantize(_rows(1100, 300, torch.float32, 4))]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ys = [P.mx4_matmul(x, w) for x in xs]
    for seed in range(3):
        xs[0].copy_(_rows(520, 300, torch.float32, 10 + seed))
        xs[1].copy_(_rows(520, 300, torch.bfloat16, 20 + seed))
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(y, P.mx4_matmul(x, w)) for x, y in zip(xs, ys))


def test_rows_behind_the_result_stay_as_they_were(P):
    """ldy > N: what lies between and behind the rows of y is not touched (through the C-ABI)."""
    import torch
    from paper_2602_05499_amd import binding as B
    for m, n, k in ((1, 70, 200), (5, 67, 200), (40, 130, 300), (300, 257, 300)):
        x, w = _rows(m, k, torch.float32, 1), P.mx4_quantize(_rows(n, k, torch.float32, 2))
        want = P.mx4_matmul(x, w)
        y = torch.full((m + 2, n + 3), 7.5, device="cuda")
        assert B.sd_mx4_matmul(w.data.data_ptr(), w.data.numel(), n, k, x.data_ptr(), B.SD_F32, k, m, None, 0.0, y.data_ptr(), B.SD_F32,
                               n + 3, torch.cuda.current_stream().cuda_stream) == B.SD_OK
        assert torch.equal(y[:m, :n], want) and (y[m:] == 7.5).all() and (y[:, n:] == 7.5).all()
        back = torch.full((n + 1, k + 5), 7.5, device="cuda")
        assert B.sd_mx4_dequantize(w.data.data_ptr(), w.data.numel(), n, k, back.data_ptr(), B.SD_F32, k + 5,
                                   torch.cuda.current_stream().cuda_stream) == B.SD_OK
        assert torch.equal(back[:n, :k], P.mx4_dequantize(w)) and (back[n:] == 7.5).all() and (back[:, k:] == 7.5).all()


def test_mismatched_tensors_are_refused(P):
    import torch
    w = P.mx4_quantize(_rows(70, 200, torch.float32, 1))
    x = _rows(3, 200, torch.float32, 2)
    bad = (lambda: P.mx4_matmul(x[:, :199], w), lambda: P.mx4_matmul(x.t(), w), lambda: P.mx4_matmul(x[0], w), lambda: P.mx4_matmul(x.half(), w),
           lambda: P.mx4_matmul(x, w, gain=x[0, :100]), lambda: P.mx4_matmul(x.bfloat16(), w, gain=x[0]), lambda: P.mx4_matmul(x.cpu(), w),
           lambda: P.mx4_matmul(x, w, gain=x[0].double()), lambda: P.mx4_matmul(x, w, out_dtype=torch.float16),
           lambda: P.mx4_matmul(x[:1].expand(3, 200), w), lambda: P.mx4_quantize(x[:, ::2]), lambda: P.mx4_quantize(x[:0]),
           lambda: P.Mx4(w.data[:-1], 70, 200), lambda: P.Mx4(w.data[16:], 1, 1), lambda: P.mx4_dequantize(w, torch.float16),
           lambda: P.mx4_matmul(x, w, gain=x[0], eps=-1.0))
    for call in bad:
        with pytest.raises(P.SdError) as e:
            call()
        assert e.value.code == P.SD_EINVAL


@pytest.mark.parametrize("m", [1, 20, 300])
def test_other_stream_and_captured_graph(P, m):
    """Calls on a side stream, and captured into a graph whose replays see the buffers' new contents each time."""
    import torch
    x, wf = _rows(m, 500, torch.float32, 1), _rows(200, 500, torch.float32, 2)
    w = P.mx4_quantize(wf)
    gain = torch.ones(500, device="cuda")
    want = P.mx4_matmul(x, w, gain=gain)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = P.mx4_matmul(x, P.mx4_quantize(wf), gain=gain)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, want)
    xin = x.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = P.mx4_matmul(P.mx4_quantize(P.mx4_matmul(xin, w, gain=gain)), P.mx4_quantize(wf[:, :200]))
    for seed in range(4):
        xin.copy_(_rows(m, 500, torch.float32, 20 + seed))
        g.replay()
        torch.cuda.synchronize()
        eager = P.mx4_matmul(P.mx4_quantize(P.mx4_matmul(xin, w, gain=gain)), P.mx4_quantize(wf[:, :200]))
        assert torch.equal(out, eager)


def test_offsets_past_32_bits(P):
    """Two million rows of 4097: more than 2^32 elements and bytes of panels; the last rows as the same rows on their own."""
    import torch
    head, cols = 2 ** 21, 4097
    x = torch.zeros(head + 70, cols, dtype=torch.bfloat16, device="cuda")
    tail = _rows(70, cols, torch.bfloat16, 4)
    x[head:] = tail
    q, qt = P.mx4_quantize(x), P.mx4_quantize(tail)
    assert q.data.numel() > 2 ** 32 and torch.equal(q.data[-qt.data.numel():], qt.data)
    few = _rows(3, cols, torch.float32, 5)
    wt = P.mx4_dequantize(qt).double()
    tol = (3 * -(-cols // 32) + 16) * 2.0 ** -23 * (few.double().abs() @ wt.abs().t()) + 1e-37
    y = P.mx4_matmul(few, q)
    assert ((y[:, head:].double() - few.double() @ wt.t()).abs() <= tol).all() and not y[:, :head].any()
    small = P.mx4_quantize(_rows(64, cols, torch.float32, 6))
    ws = P.mx4_dequantize(small).double()
    for many, tv in ((x, tail.double()), (q, wt)):
        y = P.mx4_matmul(many, small, out_dtype=torch.float32)
        tol = (3 * -(-cols // 32) + 16) * 2.0 ** -23 * (tv.abs() @ ws.abs().t()) + 1e-37
        assert ((y[head:].double() - tv @ ws.t()).abs() <= tol).all() and not y[:head].any()
    back = P.mx4_dequantize(q, torch.bfloat16)
    assert torch.equal(back[head:], P.mx4_dequantize(qt, torch.bfloat16)) and not back[:64].any()
