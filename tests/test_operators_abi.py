"""What the operators without a context refuse, decided on the host: every call here has a fault and must return its error code
before it would touch its made-up addresses.  And the panel format of MXFP4 as sizes."""
import ctypes

import pytest

from paper_2602_05499_amd import binding as B

A = 0x7F0000000000          # aligned, never read


@pytest.fixture(scope="module", autouse=True)
def lib():
    import os
    if not os.path.exists(B.library_path()):
        from paper_2602_05499_amd.session import build_library
        build_library()
    return B.load_library()


def test_sizes_of_panels():
    assert B.sd_mx4_bytes(1, 1) == 4352 and B.sd_mx4_bytes(64, 128) == 4352
    assert B.sd_mx4_bytes(65, 128) == B.sd_mx4_bytes(64, 129) == 2 * 4352
    assert B.sd_mx4_bytes(128256, 4096) == 2004 * 32 * 4352
    for r, c in ((0, 1), (1, 0), (-3, 5), (5, -3), (1, 2 ** 31 - 1)):
        assert B.sd_mx4_bytes(r, c) == 0


@pytest.mark.parametrize("over,code", [
    (dict(rows=0), B.SD_EINVAL), (dict(cols=0), B.SD_EINVAL), (dict(rows=-1), B.SD_EINVAL), (dict(x=None), B.SD_EINVAL),
    (dict(x=A + 2), B.SD_EINVAL), (dict(dtype=B.SD_BF16, x=A + 1), B.SD_EINVAL), (dict(dtype=B.SD_MX4), B.SD_EINVAL),
    (dict(dtype=-1), B.SD_EINVAL), (dict(ld=199), B.SD_EINVAL), (dict(ld=-200), B.SD_EINVAL), (dict(q=None), B.SD_EINVAL),
    (dict(q=A + 128), B.SD_EINVAL), (dict(n=2 * 2 * 4352 - 1), B.SD_ENOMEM), (dict(rows=2 ** 31 - 1, cols=2 ** 20, ld=2 ** 20), B.SD_EINVAL),
])
def test_quantize_and_dequantize_refuse(over, code):
    a = dict(x=A, dtype=B.SD_F32, ld=200, rows=70, cols=200, q=A, n=2 * 2 * 4352)
    a.update(over)
    assert B.sd_mx4_quantize(a["x"], a["dtype"], a["ld"], a["rows"], a["cols"], a["q"], a["n"], None) == code
    assert B.sd_mx4_dequantize(a["q"], a["n"], a["rows"], a["cols"], a["x"], a["dtype"], a["ld"], None) == code


@pytest.mark.parametrize("over,code", [
    (dict(w=None), B.SD_EINVAL), (dict(w=A + 16), B.SD_EINVAL), (dict(wb=2 * 2 * 4352 - 1), B.SD_ENOMEM), (dict(N=0), B.SD_EINVAL),
    (dict(K=0), B.SD_EINVAL), (dict(M=0), B.SD_EINVAL), (dict(M=-4), B.SD_EINVAL), (dict(x=None), B.SD_EINVAL),
    (dict(xt=3), B.SD_EINVAL), (dict(x=A + 2), B.SD_EINVAL), (dict(ldx=199), B.SD_EINVAL), (dict(y=None), B.SD_EINVAL),
    (dict(yt=B.SD_MX4), B.SD_EINVAL), (dict(y=A + 2), B.SD_EINVAL), (dict(ldy=69), B.SD_EINVAL),
    (dict(xt=B.SD_BF16, gain=A), B.SD_EINVAL), (dict(gain=A + 2), B.SD_EINVAL), (dict(gain=A, eps=-1.0), B.SD_EINVAL),
    (dict(gain=A, eps=float("nan")), B.SD_EINVAL), (dict(xt=B.SD_MX4, ldx=2 * 4352 - 1), B.SD_ENOMEM),
    (dict(xt=B.SD_MX4, ldx=-1), B.SD_EINVAL), (dict(xt=B.SD_MX4, x=A + 64), B.SD_EINVAL),
    (dict(xt=B.SD_MX4, gain=A), B.SD_EINVAL),
])
def test_matmul_refuses(over, code):
    a = dict(w=A, wb=2 * 2 * 4352, N=70, K=200, x=A, xt=B.SD_F32, ldx=200, M=3, gain=None, eps=1e-5, y=A, yt=B.SD_F32, ldy=70)
    if over.get("xt") == B.SD_MX4:
        a["ldx"] = 2 * 4352
    a.update(over)
    assert B.sd_mx4_matmul(a["w"], a["wb"], a["N"], a["K"], a["x"], a["xt"], a["ldx"], a["M"], a["gain"], a["eps"], a["y"], a["yt"],
                           a["ldy"], None) == code


def _rules(**over):
    a = dict(repetition=1.0, presence=0.0, frequency=0.0, bias=None, allowed=None, n_masks=0)
    a.update(over)
    return B.SdRules(*[a[n] for n, _ in B.SdRules._fields_])


@pytest.mark.parametrize("over,rules", [
    (dict(z=None), {}), (dict(out=None), {}), (dict(z=A + 2), {}), (dict(out=A + 2), {}), (dict(dtype=B.SD_MX4), {}), (dict(rows=0), {}),
    (dict(vocab=0), {}), (dict(vocab=2 ** 31 - 1, ld=2 ** 32, ld_out=2 ** 32), {}), (dict(ld=99), {}), (dict(ld_out=99), {}),
    (dict(ld_out=101, out=A), {}),                                    # in place with another distance of rows
    ({}, dict(repetition=0.0)), ({}, dict(repetition=-1.0)), ({}, dict(repetition=float("inf"))), ({}, dict(repetition=float("nan"))),
    ({}, dict(presence=float("nan"))), ({}, dict(frequency=float("inf"))), ({}, dict(bias=A + 2)), ({}, dict(allowed=A + 1, n_masks=1)),
    ({}, dict(allowed=A, n_masks=0)), ({}, dict(allowed=A, n_masks=-1)),
    ({}, dict(allowed=A, n_masks=2)),                                 # neither one mask nor one per row, and no mask_row
    (dict(mask_row=A + 2), dict(allowed=A, n_masks=2)),
    (dict(tokens=None), dict(repetition=2.0)), (dict(begin=None), dict(presence=1.0)), (dict(end=None), dict(frequency=1.0)),
    (dict(n=-1), dict(frequency=1.0)), (dict(tokens=A + 2), dict(frequency=1.0)), (dict(begin=A + 4), dict(frequency=1.0)),
    (dict(end=A + 4), dict(frequency=1.0)),
])
def test_logits_rules_refuse(over, rules):
    a = dict(z=A, dtype=B.SD_F32, ld=100, rows=3, vocab=100, tokens=A, n=10, begin=A, end=A, mask_row=None, out=A + 4096, ld_out=100)
    a.update(over)
    r = _rules(**rules)
    assert B.sd_logits_rules(a["z"], a["dtype"], a["ld"], a["rows"], a["vocab"], r, a["tokens"], a["n"], a["begin"], a["end"],
                             a["mask_row"], a["out"], a["ld_out"], None) == B.SD_EINVAL
    assert B.sd_logits_rules(A, B.SD_F32, 100, 3, 100, None, A, 10, A, A, None, A + 4096, 100, None) == B.SD_EINVAL


def test_more_than_a_launch_holds_is_refused():
    """2^32 - 1 threads: 256 per panel of a matrix, 512 per panel of outputs of a product with few rows."""
    rows = 64 * 2 ** 24
    n = B.sd_mx4_bytes(rows, 1)
    assert n == 2 ** 24 * 4352
    assert B.sd_mx4_quantize(A, B.SD_F32, 1, rows, 1, A, n, None) == B.SD_EINVAL
    assert B.sd_mx4_dequantize(A, n, rows, 1, A, B.SD_F32, 1, None) == B.SD_EINVAL
    for M, N in ((1, rows), (3, rows // 2), (16, rows // 2), (2 ** 30, 64), (2 ** 28, 1025)):
        assert B.sd_mx4_matmul(A, B.sd_mx4_bytes(N, 1), N, 1, A, B.SD_BF16, 1, M, None, 0.0, A, B.SD_F32, N, None) == B.SD_EINVAL


@pytest.mark.parametrize("dtype,es", [(B.SD_F32, 4), (B.SD_BF16, 2)])
@pytest.mark.parametrize("off", [1, 99, 229, 231, 290, 619, -1, -99, -161, -520])
def test_rows_across_rows_are_refused(dtype, es, off):
    """out as rows of 100 at distance 260, moved by off elements against z: each of these shares entries with z's three rows."""
    mine = {r * 260 + i for r in range(3) for i in range(100)}
    assert mine & {off + e for e in mine}
    z = A + (1 << 20)
    assert B.sd_logits_rules(z, dtype, 260, 3, 100, _rules(), None, 0, None, None, None, z + off * es, 260, None) == B.SD_EINVAL


def test_tensors_that_are_no_gpu_rows_are_refused():
    import torch
    import paper_2602_05499_amd as P
    for call in (lambda: P.mx4_quantize(torch.zeros(4, 64)), lambda: P.mx4_quantize(None), lambda: P.logits_rules(torch.zeros(2, 9)),
                 lambda: P.mx4_matmul(torch.zeros(2, 9), None), lambda: P.Mx4(torch.zeros(4352, dtype=torch.uint8), 1, 1),
                 lambda: P.mx4_dequantize(torch.zeros(4352, dtype=torch.uint8))):
        with pytest.raises(P.SdError) as e:
            call()
        assert e.value.code == P.SD_EINVAL
    with pytest.raises(AttributeError):
        P.no_such_operator


def test_the_rules_struct_has_the_headers_layout():
    assert [n for n, _ in B.SdRules._fields_][:3] == ["repetition", "presence", "frequency"]
    assert B.SdRules.bias.offset == 16 and B.SdRules.allowed.offset == 24 and B.SdRules.n_masks.offset == 32
    assert ctypes.sizeof(B.SdRules) == 40


def _context(**over):
    L = 2
    base = dict(n_layers=L, d_model=64, n_heads=2, n_kv_heads=2, head_dim=32, d_ffn=64, vocab=100, max_seq=64, max_k=4, dtype=B.SD_F32,
                max_out=64, rms_eps=1e-5, rope_theta=10000.0, temperature=1.0)
    base.update(over)
    cfg = B.SdConfig(*[base[n] for n, _ in B.SdConfig._fields_])
    arrs = [(ctypes.c_void_p * L)(*[A + 4096 * (i + 1) for i in range(L)]) for _ in range(9)]
    w = B.SdWeights(A, A + 256, A + 512, *[ctypes.cast(a, ctypes.POINTER(ctypes.c_void_p)) for a in arrs])
    rc, ctx = B.sd_init(cfg, w, None, A, B.sd_kv_bytes(cfg), A, B.sd_workspace_bytes(cfg), None)
    assert rc == B.SD_OK
    return cfg, ctx, arrs


def test_draft_head_is_checked_on_the_host():
    cfg, ctx, keep = _context()
    n = B.sd_mx4_bytes(cfg.vocab, cfg.d_model)
    assert B.sd_set_draft_head(ctx, A, n) == B.SD_OK and B.sd_set_draft_head(ctx, None, 0) == B.SD_OK
    assert B.sd_set_draft_head(ctx, A + 16, n) == B.SD_EINVAL
    assert B.sd_set_draft_head(ctx, A, n - 1) == B.SD_ENOMEM
    assert B.sd_set_draft_head(ctypes.c_void_p(None), A, n) == B.SD_EINVAL
    B.sd_free(ctx)


def test_context_rules_are_checked_on_the_host():
    cfg, ctx, keep = _context()
    assert B.sd_rules_bytes(cfg, -1) == 0 and B.sd_rules_bytes(None, 0) == 0
    n0, n1, n70 = (B.sd_rules_bytes(cfg, n) for n in (0, 1, 70))
    assert n0 == 512 + 256 and n1 == n0 + 256 and n70 == n0 + 512
    ok = _rules(presence=1.0)
    for call in (lambda: (ok, None, 0, None, n0), lambda: (ok, None, 0, A + 8, n0), lambda: (_rules(repetition=-1.0), None, 0, A, n0),
                 lambda: (ok, A, 0, A, n0),                                                   # next without masks
                 lambda: (_rules(allowed=A, n_masks=2), None, 0, A, n70),                     # several masks without next
                 lambda: (_rules(allowed=A, n_masks=2), A + 2, 0, A, n70),
                 lambda: (_rules(allowed=A, n_masks=2), A, 2, A, n70), lambda: (_rules(allowed=A, n_masks=2), A, -2, A, n70),
                 lambda: (_rules(allowed=A, n_masks=0), A, -1, A, n70), lambda: (_rules(bias=A + 1), None, 0, A, n0)):
        assert B.sd_set_rules(ctx, *call()) == B.SD_EINVAL
    assert B.sd_set_rules(ctx, ok, None, 0, A, n0 - 1) == B.SD_ENOMEM
    assert B.sd_set_rules(ctx, _rules(allowed=A, n_masks=70), A, 0, A, n70 - 1) == B.SD_ENOMEM
    assert B.sd_set_rules(ctx, None, None, 0, None, 0) == B.SD_OK
    assert B.sd_set_rules(ctypes.c_void_p(None), ok, None, 0, A, n0) == B.SD_EINVAL
    B.sd_free(ctx)
