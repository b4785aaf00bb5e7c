"""Every instance of the kernel for a few rows that the choice of kernel reaches, against the product in float64."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2602_05499_amd as P
    return P


def _rows(rows, cols, dtype, seed):
    import torch
    g = torch.Generator("cuda").manual_seed(seed)
    x = torch.randn(rows, cols, device="cuda", generator=g)
    return (x * torch.exp2(torch.randint(-6, 7, (rows, 1), device="cuda", generator=g).float())).to(dtype)


# Workgroups of 16 rows x 64 outputs: fewer than 128 are cut into 16-row tiles of a panel ("tile"), else a panel each ("panel"); float32 of
# 6 rows and more takes two panels each from 384 on ("two"; an odd number of panels repeats the last one).  Rows that are staged: 1,
# 5 (bfloat16 4), 8, 16; beyond 16 rows the codes are read by several workgroups.
SIZES = [("float32", 1, 1003), ("float32", 1, 8200), ("float32", 5, 1003), ("float32", 5, 24577),       # tile, panel, tile, panel
         ("float32", 6, 1003), ("float32", 7, 8200), ("float32", 8, 24577), ("float32", 8, 24700),      # tile, panel, two (odd, even)
         ("float32", 9, 1003), ("float32", 13, 8200), ("float32", 16, 24577), ("float32", 16, 24700),   # the same, 16 rows staged
         ("float32", 40, 1003), ("float32", 40, 3000), ("float32", 40, 11009), ("float32", 500, 1000),  # the same, several workgroups
         ("bfloat16", 1, 1003), ("bfloat16", 1, 8200), ("bfloat16", 4, 1003), ("bfloat16", 3, 8200),
         ("bfloat16", 6, 1003), ("bfloat16", 7, 8200), ("bfloat16", 8, 32003), ("bfloat16", 9, 1003),
         ("bfloat16", 13, 8200), ("bfloat16", 16, 32003), ("bfloat16", 40, 1003), ("bfloat16", 40, 3000),
         ("mx4", 1, 1003), ("mx4", 1, 8200), ("mx4", 5, 1003), ("mx4", 16, 8200), ("mx4", 40, 1003), ("mx4", 40, 3000)]


def _check(P, x, xv, wq, wv, m, n, k, gain=None):
    """The product within wider rows: the values (each of the at most 3 ceil(k / 32) + 16 additions of an output's chain is off by at
    most 2^-23 of a partial sum, which the sum of magnitudes bounds; bfloat16 x rounds the result once more; a norm adds k / 32 + 24
    roundings for the rows' factor), nothing beside them, the same bits again."""
    import torch
    from paper_2602_05499_amd import binding as B
    code, ptr, ld, out = ((B.SD_MX4, x.data.data_ptr(), x.data.numel(), torch.float32) if isinstance(x, P.Mx4) else
                          (B.SD_F32, x.data_ptr(), k, x.dtype) if x.dtype == torch.float32 else (B.SD_BF16, x.data_ptr(), k, x.dtype))
    y = torch.full((m + 1, n + 3), 7.5, dtype=out, device="cuda")
    assert B.sd_mx4_matmul(wq.data.data_ptr(), wq.data.numel(), n, k, ptr, code, ld, m, None if gain is None else gain.data_ptr(), 1e-5,
                           y.data_ptr(), B.SD_F32 if out == torch.float32 else B.SD_BF16, n + 3, torch.cuda.current_stream().cuda_stream) == B.SD_OK
    assert (y[m:] == 7.5).all() and (y[:, n:] == 7.5).all()
    want, mag = xv @ wv.t(), xv.abs() @ wv.abs().t()
    tol = (3 * -(-k // 32) + 16 + (0 if gain is None else k / 32 + 24)) * 2.0 ** -23 * mag + 1e-37
    if out == torch.bfloat16:
        tol = tol + 2.0 ** -8 * want.abs()
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(y[:m, :n]), nan)
    assert ((y[:m, :n].double() - want).abs() <= tol)[~nan].all()
    assert torch.equal(P.mx4_matmul(x, wq, gain=gain).nan_to_num(), y[:m, :n].nan_to_num())


@pytest.mark.parametrize("kind,m,n", SIZES)
@pytest.mark.parametrize("k", [20, 1000, 1281])
def test_every_instance(P, kind, m, n, k):
    """float32 with and without a gain; a NaN block in the last panel of w fills its output and nothing else."""
    import torch
    wf = _rows(n, k, torch.float32, n + k)
    for bad in (False, True):
        if bad:
            wf[n - 1, k - 1] = float("nan")
            wf[n // 2, 0] = float("inf")
        wq = P.mx4_quantize(wf)
        wv = P.mx4_dequantize(wq).double()
        xf = _rows(m, k, torch.float32, m + k)
        x = P.mx4_quantize(xf) if kind == "mx4" else xf.to(getattr(torch, kind))
        xv = (P.mx4_dequantize(x) if kind == "mx4" else x).double()
        _check(P, x, xv, wq, wv, m, n, k)
        if kind == "float32":
            gain = 1.0 + 0.3 * _rows(1, k, torch.float32, 3)[0].clamp(-2, 2)
            xh = xv * gain.double() / torch.sqrt((xv ** 2).mean(-1, keepdim=True) + 1e-5)
            _check(P, x, xh, wq, wv, m, n, k, gain)


@pytest.mark.parametrize("m,n", [(1, 70), (5, 8200), (16, 70), (16, 8200), (40, 70), (40, 3000)])
@pytest.mark.parametrize("k", [1000, 2048, 2049, 2300, 2560, 3100, 4097, 5120, 6200, 14336])
def test_both_sides_mxfp4_at_every_exit_of_the_loop(P, m, n, k):
    """8 waves take every eighth panel of 128 columns, two ahead: one, two or three panels left behind the steady part, which runs
    0 to 6 times.  Panels of different size, so that one taken twice or left out shows."""
    import torch
    scale = torch.exp2(torch.arange(-(-k // 128), device="cuda").remainder(5).float() - 2).repeat_interleave(128)[:k]
    wq = P.mx4_quantize(_rows(n, k, torch.float32, n + k) * scale)
    x = P.mx4_quantize(_rows(m, k, torch.float32, m + k))
    _check(P, x, P.mx4_dequantize(x).double(), wq, P.mx4_dequantize(wq).double(), m, n, k)


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
@pytest.mark.parametrize("m,n", [(1, 70), (7, 8200), (16, 8200), (7, 24577), (40, 3000)])
@pytest.mark.parametrize("k", [4097, 5120, 14336])
def test_long_reductions(P, kind, m, n, k):
    import torch
    wq = P.mx4_quantize(_rows(n, k, torch.float32, n + k))
    x = _rows(m, k, getattr(torch, kind), m + k)
    _check(P, x, x.double(), wq, P.mx4_dequantize(wq).double(), m, n, k)
