"""Panels that a caller filled, through every kernel of the product."""
import numpy as np
import pytest

from test_gpu_mx4 import GRID

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2602_05499_amd as P
    return P


# rows of x and outputs that take each kernel: few rows (one 16-row tile of a panel, a panel, two panels per workgroup; 1, 5, 8, 16
# rows staged, once or for several workgroups), then the tile kernels
ROWS = [(1, 70), (4, 70), (7, 70), (16, 70), (40, 70), (1, 8200), (7, 8200), (12, 24577), (40, 3000), (40, 11009)]
TILES = {"float32": [(129, 11009), (300, 11009), (520, 11009)], "bfloat16": [(100, 6001), (200, 11009), (520, 11009)],
         "mx4": [(100, 8003), (1100, 7777)]}
SIZES = [(t, m, n) for t in ("float32", "bfloat16", "mx4") for m, n in ROWS + TILES[t]]


@pytest.mark.parametrize("kind,m,n", SIZES)
@pytest.mark.parametrize("k", [20, 130, 300, 1185, 2200])
def test_scale_bytes_behind_the_matrix_count_for_nothing(P, kind, m, n, k):
    """Blocks past the last column or row hold zero codes; whatever their scale bytes are, 255 included, the result is the same bits."""
    import torch
    kps, blocks = -(-k // 128), -(-k // 32)
    g = torch.Generator("cuda").manual_seed(m + n + k)

    def both(rows):
        a = P.mx4_quantize(torch.randn(rows, k, device="cuda", generator=g))
        d = a.data.clone().view(-1, kps, 4352)
        scales = d[:, kps - 1, 4096:].view(-1, 4, 64)          # [panel][block][row]
        scales[:, blocks - (kps - 1) * 4:] = 255
        row = 16 * torch.arange(4, device="cuda")[None, :] + torch.arange(16, device="cuda")[:, None]      # [r][t]
        d[-1][:, 4096:].view(kps, 4, 16, 4)[:, :, row >= rows - 64 * (len(d) - 1)] = 255                 # rows behind the last
        return a, P.Mx4(d.reshape(-1), rows, k)

    w, w255 = both(n)
    assert torch.equal(P.mx4_dequantize(w), P.mx4_dequantize(w255))
    if kind == "mx4":
        x, x255 = both(m)
        want = P.mx4_matmul(x, w)
        assert torch.isfinite(want).all()
        for a, b in ((x, w255), (x255, w), (x255, w255)):
            assert torch.equal(P.mx4_matmul(a, b), want)
    else:
        x = torch.randn(m, k, device="cuda", generator=g).to(getattr(torch, kind))
        want = P.mx4_matmul(x, w)
        assert torch.isfinite(want.float()).all() and torch.equal(P.mx4_matmul(x, w255), want)


def _set(q, kps, row, block, e, codes):
    """One block of 32 columns of a row: its scale byte, and codes by column."""
    t, r = row % 64 // 16, row % 16
    p = q[(row // 64) * kps + block // 4]
    b = block % 4
    p[4096 + (b * 16 + r) * 4 + t] = e
    at = ((t * 4 + b) * 16 + r) * 16
    for i, c in codes.items():
        p[at + i // 2] = (int(p[at + i // 2]) & (0x0F if i % 2 else 0xF0)) | c << (4 * (i % 2))


def _columns(kind, m, seed=3):
    """x for the three columns that matter: multiples of powers of two that MXFP4 holds as well, zeros among them; further in
    float32 values whose second and third piece are not zero, an infinity and a NaN."""
    rng = np.random.default_rng(seed)
    x = rng.choice([0.0, 1.0, -1.0, 0.5, 3.0, -6.0], (m, 3)) * 2.0 ** -20
    if kind == "float32":
        x[m // 3, 0], x[m // 2, 1] = 2.0 ** -20 * (1 + 2.0 ** -12 + 2.0 ** -22), 2.0 ** -21 * (1 + 2.0 ** -9)
    if kind != "mx4" and m > 1:
        x[m - 1, 0], x[0, 1] = np.inf, np.nan
    return x


@pytest.mark.parametrize("kind,m,n", SIZES)
@pytest.mark.parametrize("k", [130, 1100])
def test_scale_bytes_whose_values_pass_float32(P, kind, m, n, k):
    """A value of 2^128 and more is an infinity for rows of x, and follows IEEE arithmetic from there (0 times it is NaN, whichever
    pieces x has); below, the same scale byte's values are ordinary numbers.  Two sides in MXFP4 multiply the values themselves.
    Every row has one entry, or two of the largest and an ordinary one."""
    import torch
    kps = -(-k // 128)
    q = np.zeros((-(-n // 64) * kps, 4352), np.uint8)
    q[:, 4096:] = 1
    cols = [5, 37, k - 1]
    rows = {}
    at = [0, 17, 35, 50, 63, min(69, n - 1), n // 2 // 64 * 64 + 1, n // 2 // 64 * 64 + 18, n - 3, n - 2, n - 1]
    for i, row in enumerate(dict.fromkeys(at)):
        e, col = (254, 253, 252, 251)[i % 4], cols[i % 3]
        code = (7, 4, 15, 2, 6, 3, 14)[i % 7]
        ent = {col: (e, code)}
        if i % 5 == 0:                                   # a second large entry elsewhere, and an ordinary number beside it
            ent[cols[(i + 1) % 3]] = (254, 12)
            ent[cols[(i + 2) % 3]] = (127, 3)
        rows[row] = ent
        for c, (be, bc) in ent.items():
            _set(q, kps, row, c // 32, be, {c % 32: bc})
    w = P.Mx4(torch.from_numpy(q.reshape(-1)).cuda(), n, k)
    wv = np.zeros((len(rows), 3))
    for j, ent in enumerate(rows.values()):
        for c, (e, code) in ent.items():
            wv[j, cols.index(c)] = GRID[code & 7] * (-1.0 if code & 8 else 1.0) * 2.0 ** (e - 127.0)
    back = P.mx4_dequantize(w)[list(rows)][:, cols].double().cpu().numpy()
    with np.errstate(over="ignore"):
        seen = wv.astype(np.float32).astype(np.float64)
    assert np.array_equal(back, seen)
    xc = _columns(kind, m)
    x = torch.zeros(m, k, dtype=torch.float64)
    x[:, cols] = torch.from_numpy(xc)
    x = x.float().cuda()
    xc = x[:, cols].double().cpu().numpy()
    if kind == "mx4":
        x = P.mx4_quantize(x)
        assert np.array_equal(P.mx4_dequantize(x)[:, cols].double().cpu().numpy(), xc)
        seen = wv
    elif kind == "bfloat16":
        x = x.bfloat16()
        xc = x[:, cols].double().cpu().numpy()

    def product(xs):
        """Columns of zeros count too: an infinite or NaN x against a zero weight is NaN, a zero x against an infinite weight too."""
        with np.errstate(invalid="ignore", over="ignore"):
            return (xs[:, None, :] * seen[None]).sum(-1).astype(np.float32)

    other = np.ones(n, bool)
    other[list(rows)] = False
    got = P.mx4_matmul(x, w, out_dtype=torch.float32).cpu().numpy()
    want = product(xc)
    fin = np.isfinite(want)                              # at most 8 additions of what is not zero, each off by at most 2^-23
    assert np.array_equal(got[:, list(rows)][~fin], want[~fin], equal_nan=True)
    mag = (np.abs(np.nan_to_num(xc, posinf=0.0, neginf=0.0))[:, None, :] * np.where(np.isfinite(seen), np.abs(seen), 0.0)[None]).sum(-1)
    assert (np.abs(got[:, list(rows)][fin] - want[fin].astype(np.float64)) <= 8 * 2.0 ** -23 * mag[fin]).all()
    odd = ~np.isfinite(xc).all(-1)
    assert (got[~odd][:, other] == 0).all() and np.isnan(got[odd][:, other]).all()
    if kind == "float32":
        gain = torch.linspace(0.5, 1.5, k, device="cuda")
        g = gain.double().cpu().numpy()[cols]
        got = P.mx4_matmul(x, w, gain=gain, eps=1e-5).cpu().numpy()[:, list(rows)]
        with np.errstate(invalid="ignore", over="ignore"):
            want = product(xc * g / np.sqrt((xc ** 2).sum(-1, keepdims=True) / k + 1e-5))
        fin = np.isfinite(want)
        assert np.array_equal(got[~fin], want[~fin], equal_nan=True)
        assert np.isfinite(got[fin]).all()
