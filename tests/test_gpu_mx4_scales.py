"""Panels that a caller filled, through every kernel of the product."""
import pytest

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
def test_scale_bytes_behind_the_last_column_count_for_nothing(P, kind, m, n, k):
    """Blocks past the matrix hold zero codes; whatever their scale bytes are, 255 included, the result is the same bits."""
    import torch
    kps, blocks = -(-k // 128), -(-k // 32)
    g = torch.Generator("cuda").manual_seed(m + n + k)

    def both(rows):
        a = P.mx4_quantize(torch.randn(rows, k, device="cuda", generator=g))
        d = a.data.clone().view(-1, kps, 4352)
        scales = d[:, kps - 1, 4096:].view(-1, 4, 64)          # [panel][block][row]
        scales[:, blocks - (kps - 1) * 4:] = 255
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
