"""Rules on logits against a plain implementation in 64 bits: one entry to large vocabularies around the edges of the chunks a
row is cut into, empty, shared and ragged histories, foreign token ids, masks that allow nothing, infinities and NaN."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2602_05499_amd as P
    return P


def rules64(z, tokens, begin, end, rep, pres, freq, bias, allowed, mask_row):
    """(result, magnitude that bounds every intermediate value) in float64."""
    rows, vocab = z.shape
    z = z.astype(np.float64).copy()
    mag = np.abs(z)
    for r in range(rows):
        if tokens is not None:
            b, e = max(0, begin[r]), min(end[r], len(tokens))
            h = tokens[b:e] if e > b else tokens[:0]
            n = np.bincount(h[(h >= 0) & (h < vocab)], minlength=vocab)
            hit = n > 0
            pos = hit & (z[r] > 0)
            neg = hit & ~(z[r] > 0)
            z[r][pos] /= rep
            z[r][neg] *= rep
            mag[r] = np.maximum(mag[r], np.abs(z[r])) + (np.abs(freq) * n + np.abs(pres)) * hit
            z[r][hit] -= (freq * n + pres)[hit]
        if bias is not None:
            z[r] += bias
            mag[r] += np.abs(bias)
        if allowed is not None:
            m = mask_row[r] if mask_row is not None else (0 if len(allowed) == 1 else r)
            if 0 <= m < len(allowed):
                ok = np.unpackbits(allowed[m].view(np.uint8), bitorder="little")[:vocab]
                z[r][ok == 0] = -np.inf
    return z, mag


def _run(P, z, tokens=None, begin=None, end=None, rep=1.0, pres=0.0, freq=0.0, bias=None, allowed=None, mask_row=None, out=None):
    import torch
    dev = lambda a, t: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(t).cuda()   # noqa: E731
    return P.logits_rules(z, dev(tokens, torch.int32), dev(begin, torch.int64), dev(end, torch.int64), repetition=rep, presence=pres,
                          frequency=freq, bias=dev(bias, torch.float32), allowed=dev(allowed, torch.int32), mask_row=dev(mask_row, torch.int32),
                          out=out)


def _check(got, want, mag, bf16):
    """Five float32 operations, each off by at most 2^-24 of a magnitude that mag bounds (the product frequency * n counts for
    one more); bfloat16 rounds the result once more, by at most 2^-8 of it."""
    got = got.double().cpu().numpy()
    fin = np.isfinite(want)
    assert np.array_equal(got[~fin], want[~fin], equal_nan=True)
    tol = 6 * 2.0 ** -24 * mag + (2.0 ** -8 * np.abs(want) if bf16 else 0.0)
    assert (np.abs(got - want)[fin] <= tol[fin]).all()


def _case(rows, vocab, dtype, seed, hist=300, n_masks=None):
    import torch
    rng = np.random.default_rng(seed)
    z = torch.from_numpy((3 * rng.standard_normal((rows, vocab))).astype(np.float32)).to(getattr(torch, dtype)).cuda()
    tokens = (vocab * rng.random(hist) ** 3).astype(np.int32)
    begin = rng.integers(0, hist, rows)
    end = np.minimum(hist, begin + rng.integers(0, hist, rows))
    bias = np.where(rng.random(vocab) < 0.3, rng.standard_normal(vocab), 0.0).astype(np.float32)
    allowed = rng.integers(-2 ** 31, 2 ** 31, (n_masks or rows, -(-vocab // 32))).astype(np.int32)
    return z, tokens, begin, end, bias, allowed


@pytest.mark.parametrize("rows,vocab", [(1, 1), (1, 31), (3, 33), (2, 1023), (2, 1024), (5, 1025), (1, 32003), (9, 8193), (1, 131072),
                                        (140, 32003), (600, 4097), (520, 1000)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_all_rules(P, rows, vocab, dtype):
    z, tokens, begin, end, bias, allowed = _case(rows, vocab, dtype, rows + vocab)
    zn = z.double().cpu().numpy()
    bf = dtype == "bfloat16"
    for kw in (dict(rep=1.25, pres=0.5, freq=0.125, bias=bias, allowed=allowed), dict(rep=0.8, pres=-0.3, freq=-0.01), dict(freq=0.7),
               dict(pres=0.4), dict(bias=bias), dict(allowed=allowed), dict(allowed=allowed[:1]), dict()):
        f32 = {k: float(np.float32(v)) for k, v in kw.items() if k in ("rep", "pres", "freq")}
        want, mag = rules64(zn, tokens if f32 else None, begin, end, f32.get("rep", 1.0), f32.get("pres", 0.0), f32.get("freq", 0.0),
                            kw.get("bias"), kw.get("allowed"), None)
        _check(_run(P, z, tokens, begin, end, **kw), want, mag, bf)


def test_histories_empty_shared_foreign_and_out_of_range(P):
    """Rows whose ranges are empty, reversed, overlapping or past the token list; ids below 0 and past the vocabulary; one token
    many times."""
    import torch
    vocab = 2050
    rng = np.random.default_rng(1)
    z = torch.from_numpy(rng.standard_normal((8, vocab)).astype(np.float32)).cuda()
    tokens = rng.integers(-5, vocab + 5, 5001).astype(np.int32)
    tokens[:3] = (-1, -2 ** 31, 2 ** 31 - 1)
    tokens[100:3000] = 1024
    begin = np.array([0, 10, 4000, 20, 5001, -7, 0, 99])
    end = np.array([5001, 10, 2 ** 40, 10, 6000, 50, 1, 3001])
    want, mag = rules64(z.double().cpu().numpy(), tokens, begin, end, 1.25, 0.5, 0.25, None, None, None)
    _check(_run(P, z, tokens, begin, end, rep=1.25, pres=0.5, freq=0.25), want, mag, False)
    assert torch.equal(_run(P, z, tokens[:0], begin, end, rep=1.25), z)      # no tokens at all
    far = np.full(8, 2 ** 63 - 1)                                             # ranges at the ends of 64 bits
    assert torch.equal(_run(P, z, tokens, far, far, rep=1.25), z) and torch.equal(_run(P, z, tokens, far, -far, rep=1.25), z)
    want, mag = rules64(z.double().cpu().numpy(), tokens, np.zeros(8, int), np.full(8, 5001), 1.25, 0.5, 0.25, None, None, None)
    _check(_run(P, z, tokens, -far, far, rep=1.25, pres=0.5, freq=0.25), want, mag, False)


def test_masks_per_row(P):
    import torch
    vocab = 100
    z = torch.randn(5, vocab, device="cuda")
    allowed = np.zeros((3, 4), np.int32)
    allowed[1] = -1
    allowed[2, 3] = 1 << 3                                # token 99 alone
    got = _run(P, z, allowed=allowed, mask_row=np.array([0, 1, 2, -1, 3])).cpu()
    zc = z.cpu()
    assert torch.isneginf(got[0]).all()                   # a mask that allows nothing
    assert torch.equal(got[1], zc[1]) and torch.equal(got[3], zc[3]) and torch.equal(got[4], zc[4])
    assert torch.isneginf(got[2, :99]).all() and got[2, 99] == zc[2, 99]


def test_infinities_nan_and_lowest_values(P):
    """-inf logits stay, NaN stays where it is allowed and goes where it is masked, a bias of the type's lowest value or -inf is
    an ordinary addition."""
    import torch
    vocab = 64
    z = torch.zeros(1, vocab, device="cuda")
    z[0, 0], z[0, 1], z[0, 2], z[0, 3], z[0, 4] = float("-inf"), float("inf"), float("nan"), float("nan"), 1.0
    bias = np.zeros(vocab, np.float32)
    bias[5], bias[6], bias[7] = -np.inf, np.finfo(np.float32).min, np.finfo(np.float32).min
    z[0, 7] = torch.finfo(torch.float32).min
    allowed = np.full((1, 2), -1, np.int32)
    allowed[0, 0] = ~(1 << 3)
    got = _run(P, z, np.arange(8, dtype=np.int32), [0], [8], rep=2.0, pres=1.0, bias=bias, allowed=allowed)[0].cpu()
    assert got[0] == float("-inf") and got[1] == float("inf") and torch.isnan(got[2]) and got[3] == float("-inf") and got[4] == -0.5
    assert got[5] == float("-inf") and got[6] == np.finfo(np.float32).min and got[7] == float("-inf")
    assert (got[8:] == 0).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_in_place_strided_and_behind_the_rows(P, dtype):
    import torch
    z, tokens, begin, end, bias, allowed = _case(6, 1111, dtype, 3)
    kw = dict(tokens=tokens, begin=begin, end=end, rep=1.3, pres=0.1, freq=0.2, bias=bias, allowed=allowed)
    want = _run(P, z, **kw)
    big = torch.full((8, 1200), 9.0, dtype=z.dtype, device="cuda")
    view = big[1:7, 3:1114]
    view.copy_(z)
    assert torch.equal(_run(P, view, **kw), want)
    assert _run(P, view, out=view, **kw) is view and torch.equal(view, want)
    big[1:7, 3:1114] = 9.0
    assert (big == 9.0).all()
    out = torch.full((6, 1113), 5.0, dtype=z.dtype, device="cuda")
    _run(P, z, out=out[:, 1:1112], **kw)
    assert torch.equal(out[:, 1:1112], want) and (out[:, 0] == 5.0).all() and (out[:, 1112] == 5.0).all()


def test_refusals(P):
    import torch
    z = torch.zeros(3, 100, device="cuda")
    i32, i64 = dict(dtype=torch.int32, device="cuda"), dict(dtype=torch.int64, device="cuda")
    t, b, m = torch.zeros(5, **i32), torch.zeros(3, **i64), torch.zeros(3, 4, **i32)
    for call in (lambda: P.logits_rules(z, repetition=2.0), lambda: P.logits_rules(z, t, b, repetition=2.0),
                 lambda: P.logits_rules(z, t.long(), b, b, presence=1.0), lambda: P.logits_rules(z, t, b.int(), b, presence=1.0),
                 lambda: P.logits_rules(z, t, b[:2], b, presence=1.0), lambda: P.logits_rules(z, t.cpu(), b, b, presence=1.0),
                 lambda: P.logits_rules(z, bias=z[0, :99]), lambda: P.logits_rules(z, bias=z[0].double()),
                 lambda: P.logits_rules(z, allowed=m[:, :3].contiguous()), lambda: P.logits_rules(z, allowed=m[:2]),
                 lambda: P.logits_rules(z, allowed=m.long()), lambda: P.logits_rules(z, allowed=m, mask_row=b),
                 lambda: P.logits_rules(z, t, b, b, repetition=0.0), lambda: P.logits_rules(z, t, b, b, frequency=float("nan")),
                 lambda: P.logits_rules(z.half()), lambda: P.logits_rules(z[0]), lambda: P.logits_rules(z.t()),
                 lambda: P.logits_rules(z, out=z[:2]), lambda: P.logits_rules(z, out=z.bfloat16()), lambda: P.logits_rules(z[:1].expand(3, 100))):
        with pytest.raises(P.SdError) as e:
            call()
        assert e.value.code == P.SD_EINVAL


def test_rows_between_rows_and_refused_overlaps(P):
    """z and out may lie between one another's rows, never across them; no masks at all is no rule but a mistake."""
    import torch
    buf = torch.randn(3, 260, device="cuda", generator=torch.Generator("cuda").manual_seed(8))
    z, before = buf[:, :100], buf.clone()
    bias = torch.linspace(-2, 2, 100, device="cuda")
    for at in (100, 130, 160):
        out = P.logits_rules(z, bias=bias, out=buf[:, at:at + 100])
        assert torch.equal(out, before[:, :100] + bias) and torch.equal(z, before[:, :100])
    flat = buf.view(-1)
    for bad in (dict(out=buf[:, 1:101]), dict(out=flat[200:720].view(2, 260)[:, :100]), dict(allowed=torch.zeros(0, 4, dtype=torch.int32, device="cuda"))):
        with pytest.raises(P.SdError) as e:
            P.logits_rules(z[:bad["out"].shape[0]] if "out" in bad else z, **bad)
        assert e.value.code == P.SD_EINVAL


def test_more_rows_than_an_int_are_refused(P):
    """Sizes are 32-bit: 2^32 + 5 rows must not be taken for 5."""
    import torch
    z = torch.empty(2 ** 32 + 5, 1, dtype=torch.bfloat16, device="cuda")
    w = P.mx4_quantize(torch.ones(1, 1, device="cuda"))
    for call in (lambda: P.logits_rules(z, out=z), lambda: P.mx4_quantize(z), lambda: P.mx4_matmul(z, w), lambda: P.mx4_quantize(z.view(1, -1)),
                 lambda: P.Mx4(w.data, 2 ** 32 + 1, 1)):
        with pytest.raises(P.SdError) as e:
            call()
        assert e.value.code == P.SD_EINVAL


def test_other_stream_and_captured_graph(P):
    import torch
    z, tokens, begin, end, bias, allowed = _case(4, 5000, "float32", 9)
    dev = [torch.from_numpy(tokens).cuda(), torch.from_numpy(begin).cuda(), torch.from_numpy(end).cuda()]
    kw = dict(repetition=1.2, presence=0.1, frequency=0.3, bias=torch.from_numpy(bias).cuda(), allowed=torch.from_numpy(allowed).cuda())
    want = P.logits_rules(z, *dev, **kw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = P.logits_rules(z, *dev, **kw)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = P.logits_rules(z, *dev, **kw)
    for i in range(4):
        z.normal_()
        dev[0].random_(0, 5000)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, P.logits_rules(z, *dev, **kw))


def test_offsets_past_32_bits(P):
    """9 GB of logits in place: the last rows, four billion entries in, as the same rows on their own."""
    import torch
    rows, vocab = 70000, 65537
    z = torch.zeros(rows, vocab, dtype=torch.bfloat16, device="cuda")
    z[-3:] = torch.randn(3, vocab, device="cuda", generator=torch.Generator("cuda").manual_seed(3)).bfloat16()
    bias = torch.linspace(-3, 3, vocab, device="cuda")
    allowed = torch.full((1, -(-vocab // 32)), 0x5A5A5A5A, dtype=torch.int32, device="cuda")
    tokens = torch.arange(0, vocab, 7, dtype=torch.int32, device="cuda")
    begin = torch.zeros(rows, dtype=torch.int64, device="cuda")
    kw = dict(repetition=1.25, presence=0.5, bias=bias, allowed=allowed)
    end = torch.zeros_like(begin)
    end[-2:] = tokens.numel()
    want = P.logits_rules(z[-3:].clone(), tokens, begin[-3:], end[-3:].clone(), **kw)
    first = P.logits_rules(z[:1].clone(), tokens, begin[:1], end[:1], **kw)
    assert P.logits_rules(z, tokens, begin, end, out=z, **kw) is z
    assert torch.equal(z[-3:], want) and torch.equal(z[:1], first) and torch.equal(z[rows // 2:rows // 2 + 1], first)


@pytest.mark.parametrize("rows,vocab", [(2 ** 24 + 77, 3), (2 ** 23 + 5, 4097)])
def test_more_rows_than_a_launch_holds(P, rows, vocab):
    """16777215 workgroups of 256 threads are a launch; rows past them, masks by row and histories among them, come in the next."""
    import torch
    z = torch.zeros(rows, vocab, dtype=torch.bfloat16, device="cuda")
    i = torch.arange(rows, device="cuda")
    z[:, 0] = (i % 251).bfloat16()
    tokens = torch.tensor([0, 0, 1], dtype=torch.int32, device="cuda")
    end = torch.where(i % 3 == 0, 3, 0)
    allowed = torch.tensor([[-1], [-3]], dtype=torch.int32, device="cuda").expand(2, -(-vocab // 32)).contiguous()
    got = P.logits_rules(z, tokens, torch.zeros_like(i), end, frequency=0.5, presence=1.0, allowed=allowed,
                         mask_row=(i % 2).int(), out=z)
    hit = (i % 3 == 0).float()
    first, second = (i % 251).float() - 2.0 * hit, torch.where(i % 2 == 1, -float("inf"), -1.5 * hit)
    assert torch.equal(got[:, 0], first.bfloat16()) and torch.equal(got[:, 1], second.bfloat16()) and not got[:, 2].any()
