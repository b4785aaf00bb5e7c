"""Cases of the operators between the last hidden row and the next token: MXFP4 quantisation, the product with MXFP4
weights, and the rules on logits (penalties for repeated tokens, biases, grammar masks).

Three kinds of call:

* `quantize`  rows to MXFP4 (blocks of 32 columns, 4-bit e2m1 values, one power-of-two scale per block) and back;
* `matmul`    y = x W^T with W in MXFP4: x in float32 (optionally RMS-normalised with a gain, as in front of an output
              head), in bfloat16, or in MXFP4 as well;
* `rules`     rows of logits under repetition, presence and frequency penalties from token histories, a bias and bit
              masks of allowed tokens.

An MXFP4 matrix lies in panels of 64 rows x 128 columns, [ceil(rows / 64)][ceil(cols / 128)][4352] bytes: 4096 bytes of
codes, where row 16 t + r and block b of 32 columns of the panel have their 16 bytes at ((t * 4 + b) * 16 + r) * 16 (column
2 i of the block in the low four bits of byte i, 2 i + 1 in the high ones), then 256 bytes of scales, that block's at
4096 + (b * 16 + r) * 4 + t, as an exponent with bias 127.  Rows and columns past the matrix hold zeros.
"""
import math
from types import SimpleNamespace

import numpy as np
import torch

own = False          # False: the plain forms below; True: the framework's operators

DEVICE = "cuda:0"
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)   # e2m1 values, by their three low bits
PANEL = 4352
EPS = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _quantize(name, rows, cols, dtype):
    return {"name": name, "kind": "quantize", "rows": rows, "cols": cols, "dtype": dtype}


def _matmul(name, m, n, k, x, gain=False):
    return {"name": name, "kind": "matmul", "m": m, "n": n, "k": k, "x": x, "gain": gain}


def _rules(name, rows, vocab, dtype, history, shared, bias=True, mask=0.5, penalties=True):
    return {"name": name, "kind": "rules", "rows": rows, "vocab": vocab, "dtype": dtype, "history": history, "shared": shared,
            "bias": bias, "mask": mask, "penalties": penalties}


def listed():
    return [
        # the activations of a few rows with a ragged width: latency
        _quantize("quantize-5x1000", 5, 1000, "f32"),
        # an output head of the 7B shape, quantised once when a draft is made from a model
        _quantize("quantize-head-7b", 32000, 4096, "bf16"),
        # the output head behind one draft row: final norm and product (7B and the large vocabulary of Llama-3-8B's shape)
        _matmul("head-7b-1row", 1, 32000, 4096, "f32", gain=True),
        _matmul("head-l3-8b-1row", 1, 128256, 4096, "f32", gain=True),
        # the head behind the seven rows of a verify forward, 13B widths, bfloat16 rows
        _matmul("head-13b-7rows", 7, 32000, 5120, "bf16"),
        # a small projection of a narrow model over a short ragged prompt
        _matmul("small-37rows", 37, 1003, 777, "f32"),
        # gate or up projection of the 7B shape over a 512-token prompt
        _matmul("gate-7b-512rows", 512, 11008, 4096, "bf16"),
        # the largest: up projection of Llama-3-8B's shape over a 4096-token prompt, both sides in MXFP4
        _matmul("up-l3-8b-4096rows", 4096, 14336, 4096, "mx4"),
        # one draft row of a chat in full swing under all rules
        _rules("rules-1x32000", 1, 32000, "f32", 700, True),
        # the five rows of a verify forward over a long document, large vocabulary, a grammar that allows few tokens
        _rules("rules-5x128256", 5, 128256, "f32", 4100, True, mask=0.01),
        # a batch of sequences with ragged histories of their own, bfloat16 logits of an odd vocabulary
        _rules("rules-256x32003", 256, 32003, "bf16", 1500, False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(c):
    """A rough time, to keep drawn cases below the largest listed one."""
    w = work(c)
    return w["bytes"] / 4e12 + w["flops"] / 1e15


def draw(rng):
    """One more case of the same ranges; sizes spread over their logarithm, odd ones among them."""
    limit = max(_cost(c) for c in listed())
    while True:
        kind = rng.choice(["quantize", "matmul", "matmul", "matmul", "rules", "rules"])
        if kind == "quantize":
            c = _quantize("", _log_int(rng, 1, 131072), _log_int(rng, 20, 16384), rng.choice(["f32", "bf16"]))
        elif kind == "matmul":
            x = rng.choice(["f32", "f32", "bf16", "mx4"])
            few = rng.random() < 0.5                       # decode-time rows or a prompt's
            c = _matmul("", rng.randint(1, 16) if few else _log_int(rng, 17, 4096), _log_int(rng, 64, 131072),
                        _log_int(rng, 64, 16384), x, gain=x == "f32" and rng.random() < 0.5)
        else:
            shared = rng.random() < 0.5                    # the rows of one step, or a batch of sequences
            c = _rules("", rng.randint(1, 9) if shared else _log_int(rng, 2, 512), _log_int(rng, 500, 131072),
                       rng.choice(["f32", "f32", "bf16"]), _log_int(rng, 1, 16384 if shared else 4096), shared,
                       bias=rng.random() < 0.5, mask=rng.choice([0.0, 0.01, 0.5, 0.95]), penalties=rng.random() < 0.8)
            if not (c["bias"] or c["mask"] or c["penalties"]):
                continue
        del c["name"]
        if _cost(c) <= limit:
            return c


def _panels(rows, cols):
    return -(-rows // 64) * -(-cols // 128)


def work(case):
    c = case
    if c["kind"] == "quantize":
        # reads the rows, writes the panels, reads them back, writes the values they stand for (the panels are small
        # beside the rows: counted once)
        n = c["rows"] * c["cols"]
        return {"bytes": 2 * n * (4 if c["dtype"] == "f32" else 2) + n * 17 // 32, "flops": 0}
    if c["kind"] == "matmul":
        m, n, k = c["m"], c["n"], c["k"]
        x, y = {"f32": (4, 4), "bf16": (2, 2), "mx4": (17 / 32, 4)}[c["x"]]
        return {"bytes": int(n * k * 17 / 32 + m * k * x + m * n * y), "flops": 2 * m * n * k}
    e, v, r = (4 if c["dtype"] == "f32" else 2), c["vocab"], c["rows"]
    tokens = c["history"] * (1 if c["shared"] else r) if c["penalties"] else 0
    masks = (1 if c["shared"] else r) * -(-v // 32) * 4 if c["mask"] else 0
    return {"bytes": 2 * r * v * e + tokens * 4 + masks + (4 * v if c["bias"] else 0), "flops": 8 * r * v}


# ---- MXFP4 in elementary operations --------------------------------------------------------------------------------------
def _codes(x):
    """Codes (uint8, one per value) and scale exponents (uint8, one per block of 32) of float32 rows, the columns padded to
    128: the scale is the power of two of the block's largest magnitude over 4, at least 2^-126; a value is rounded to the
    nearest grid value, halfway to the one with the even code, and 6 at most."""
    rows, cols = x.shape
    x = torch.nn.functional.pad(x, (0, -cols % 128)).view(rows, -1, 32)
    amax = x.abs().amax(-1)
    e = torch.clamp(torch.frexp(amax)[1] + (126 - 2), min=1)          # frexp: amax = m 2^e with m in [1/2, 1)
    e = torch.where(amax == 0, torch.ones_like(e), e)
    a = torch.ldexp(x.abs(), (127 - e)[..., None])
    code = torch.zeros(a.shape, dtype=torch.uint8, device=x.device)
    for i in range(7):                                               # past the midpoint, or on it when the upper code is even
        mid = (GRID[i] + GRID[i + 1]) / 2
        code += (a >= mid) if i % 2 else (a > mid)
    code += 8 * torch.signbit(x).to(torch.uint8)
    return code.view(rows, -1), e.to(torch.uint8)


def _pack(code, e):
    """The panels of codes [rows][cols padded to 128] and scales [rows][cols / 32]."""
    rows, cols = code.shape
    pad = -rows % 64
    code = torch.nn.functional.pad(code, (0, 0, 0, pad)).view(-1, 4, 16, cols // 128, 4, 16, 2)
    by = (code[..., 0] | (code[..., 1] << 4)).permute(0, 3, 1, 4, 2, 5).reshape(-1, cols // 128, 4096)
    sc = torch.nn.functional.pad(e, (0, 0, 0, pad)).view(-1, 4, 16, cols // 128, 4).permute(0, 3, 4, 2, 1)
    return torch.cat([by, sc.reshape(-1, cols // 128, 256)], -1).contiguous().view(-1)


def _values(q, rows, cols):
    """The float32 values that panels stand for."""
    kp = -(-cols // 128)
    q = q.view(-1, kp, PANEL)
    table = torch.tensor(GRID + tuple(-g for g in GRID), device=q.device)
    pairs = torch.stack([table.repeat(16), table.repeat_interleave(16)], -1)       # a byte's two values
    v = pairs[q[..., :4096].int()].view(-1, kp, 4, 4, 16, 32)                      # [panel][k][t][b][r][column]
    e = q[..., 4096:].reshape(-1, kp, 4, 16, 4).permute(0, 1, 4, 2, 3)             # [panel][k][t][b][r]
    v = v * torch.ldexp(torch.ones((), device=q.device), e.int() - 127)[..., None]
    return v.permute(0, 2, 4, 1, 3, 5).reshape(-1, kp * 128)[:rows, :cols]


# ---- inputs ----------------------------------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _quantized(rows, cols, std, gen):
    """A matrix of normal values in MXFP4, made in pieces of whole panels."""
    got = []
    for r in range(0, rows, 16384):
        x = torch.empty(min(16384, rows - r), cols, device=DEVICE).normal_(0.0, std, generator=gen)
        got.append(_pack(*_codes(x)))
    return torch.cat(got)


def _rows(m, k, gen):
    """Rows of a residual stream: normal values, a few columns that stand out by a factor of ten, rows of different size."""
    x = torch.randn(m, k, device=DEVICE, generator=gen)
    x[:, torch.randint(0, k, (1 + k // 100,), device=DEVICE, generator=gen)] *= 10.0
    return x * (0.5 + torch.rand(m, 1, device=DEVICE, generator=gen))


def prepare(case, seed):
    c, gen = case, _gen(seed)
    st = SimpleNamespace(case=c)
    if c["kind"] == "quantize":
        st.x = _rows(c["rows"], c["cols"], gen).to(TYPES[c["dtype"]])
    elif c["kind"] == "matmul":
        st.w = _quantized(c["n"], c["k"], 1.0 / math.sqrt(c["k"]), gen)
        st.gain = 1.0 + 0.1 * torch.randn(c["k"], device=DEVICE, generator=gen) if c["gain"] else None
        x = _rows(c["m"], c["k"], gen)
        st.x = _pack(*_codes(x)) if c["x"] == "mx4" else x.to(TYPES[c["x"]])
    else:
        r, v = c["rows"], c["vocab"]
        st.z = (3.0 * torch.randn(r, v, device=DEVICE, generator=gen)).to(TYPES[c["dtype"]])
        st.tokens = st.begin = st.end = st.bias = st.allowed = st.mask_row = None
        if c["penalties"]:
            # texts repeat themselves: tokens by a power law, some of them very often
            n = c["history"]
            if c["shared"]:                    # the rows of one step: a history and one token more for each row
                begin, end = [0] * r, [n + i for i in range(r)]
            else:                              # sequences with histories of their own, from one token to n
                rng = np.random.default_rng(seed)
                length = np.maximum(1, (n * rng.random(r)).astype(np.int64))
                length[0] = n
                end = np.cumsum(length)
                begin = end - length
            st.begin = torch.tensor(np.asarray(begin), dtype=torch.int64, device=DEVICE)
            st.end = torch.tensor(np.asarray(end), dtype=torch.int64, device=DEVICE)
            u = torch.rand(int(max(end)), device=DEVICE, generator=gen, dtype=torch.float64)
            st.tokens = (v * u ** 3).to(torch.int32).clamp_(max=v - 1)
        if c["bias"]:                          # a few tokens are favoured or discouraged
            st.bias = torch.where(torch.rand(v, device=DEVICE, generator=gen) < 0.02, 4.0 * torch.randn(v, device=DEVICE, generator=gen),
                                  torch.zeros(v, device=DEVICE))
        if c["mask"]:                          # a grammar's allowed tokens: one state for all rows, or one for each
            n_masks = 1 if c["shared"] else r
            words = -(-v // 32)
            bits = torch.rand(n_masks, words, 32, device=DEVICE, generator=gen) < c["mask"]
            st.allowed = (bits.long() << torch.arange(32, device=DEVICE)).sum(-1).to(torch.uint32).view(torch.int32)
            st.mask_row = (torch.zeros(r, device=DEVICE) if c["shared"] else torch.randperm(r, device=DEVICE, generator=gen)).to(torch.int32)
        st.repetition, st.presence, st.frequency = (1.25, 0.5, 0.125) if c["penalties"] else (1.0, 0.0, 0.0)
    return st


# ---- the operators ---------------------------------------------------------------------------------------------------------
def _run_own(st):
    import paper_2602_05499_amd as P
    c = st.case
    if c["kind"] == "quantize":
        return P.mx4_dequantize(P.mx4_quantize(st.x), st.x.dtype)
    if c["kind"] == "matmul":
        x = P.Mx4(st.x, c["m"], c["k"]) if c["x"] == "mx4" else st.x
        return P.mx4_matmul(x, P.Mx4(st.w, c["n"], c["k"]), gain=st.gain, eps=EPS)
    return P.logits_rules(st.z, st.tokens, st.begin, st.end, repetition=st.repetition, presence=st.presence,
                          frequency=st.frequency, bias=st.bias, allowed=st.allowed, mask_row=st.mask_row)


def _counts(st, rows, vocab):
    """Occurrences of every token in every row's history."""
    n = st.end - st.begin
    row = torch.repeat_interleave(torch.arange(rows, device=DEVICE), n)
    at = torch.arange(row.numel(), device=DEVICE) - (torch.cumsum(n, 0) - n)[row] + st.begin[row]
    flat = torch.zeros(rows * vocab, dtype=torch.int32, device=DEVICE)
    return flat.scatter_add_(0, row * vocab + st.tokens[at], torch.ones_like(at, dtype=torch.int32)).view(rows, vocab)


def run(state):
    if own:
        return _run_own(state)
    st, c = state, state.case
    if c["kind"] == "quantize":
        return _values(_pack(*_codes(st.x.float())), c["rows"], c["cols"]).to(st.x.dtype)
    if c["kind"] == "matmul":
        w = _values(st.w, c["n"], c["k"])
        x = _values(st.x, c["m"], c["k"]) if c["x"] == "mx4" else st.x.float()
        if st.gain is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * st.gain
        return (x @ w.t()).to(torch.bfloat16 if c["x"] == "bf16" else torch.float32)
    z = st.z.float()
    if st.tokens is not None:
        n = _counts(st, *z.shape)
        seen = n > 0
        z = torch.where(seen, torch.where(z > 0, z / st.repetition, z * st.repetition), z)
        z = z - st.frequency * n - st.presence * seen
    if st.bias is not None:
        z = z + st.bias
    if st.allowed is not None:
        bit = torch.arange(c["vocab"], device=DEVICE)
        ok = (st.allowed[st.mask_row][:, bit // 32] >> (bit % 32)) & 1
        z = torch.where(ok == 1, z, torch.full_like(z, -math.inf))
    return z.to(st.z.dtype)


# ---- from the definitions, in 64 bits ----------------------------------------------------------------------------------------
def _exact_values(q, rows, cols):
    """The values of panels, row tile by row tile, from the bits of each code: (-1)^s (m / 2 + [e > 0]) 2^max(e - 1, 0)."""
    kp = -(-cols // 128)
    q = q.view(-1, kp, PANEL)
    out = torch.empty(q.shape[0] * 64, kp * 128, dtype=torch.float64, device=q.device)
    for t in range(4):
        by = q[:, :, 1024 * t:1024 * (t + 1)].reshape(-1, kp, 4, 16, 16).int()     # [panel][k][b][r][byte]
        scale = torch.exp2(q[:, :, 4096 + t::4].reshape(-1, kp, 4, 16).double() - 127.0)
        for odd in (0, 1):
            bits = by >> 4 if odd else by & 15
            ex = (bits >> 1) & 3
            v = ((bits & 1) * 0.5 + (ex > 0)) * torch.exp2(torch.clamp(ex - 1, min=0).double()) * (1 - 2 * (bits >> 3))
            v = (v * scale[..., None]).permute(0, 3, 1, 2, 4)                      # [panel][r][k][b][byte]
            out.view(-1, 4, 16, kp, 4, 16, 2)[:, t, :, :, :, :, odd] = v
    return out[:rows, :cols]


def _exact_quantized(x):
    """Nearest grid value of every entry: with the spacing of e2m1 at its magnitude, by rounding to even."""
    rows, cols = x.shape
    x = torch.nn.functional.pad(x.double(), (0, -cols % 32)).view(rows, -1, 32)
    amax = x.abs().amax(-1, keepdim=True)
    top = torch.floor(torch.log2(torch.where(amax > 0, amax, torch.ones_like(amax))))
    top = torch.where(torch.exp2(top) > amax, top - 1, torch.where(torch.exp2(top + 1) <= amax, top + 1, top))
    scale = torch.exp2(torch.clamp(top - 2, min=-126.0))
    a = (x / scale).abs()
    step = torch.where(a >= 4, 2.0, torch.where(a >= 2, 1.0, 0.5))                 # grid spacing: 0.5 below 2, 1, 2
    v = torch.clamp(torch.round(a / step) * step, max=6.0)
    return (torch.copysign(v, x) * scale).view(rows, -1)[:, :cols]


def exact(case, seed):
    c, st = case, prepare(case, seed)
    if c["kind"] == "quantize":
        return torch.cat([_exact_quantized(st.x[r:r + 8192]) for r in range(0, c["rows"], 8192)])
    if c["kind"] == "matmul":
        x = _exact_values(st.x, c["m"], c["k"]) if c["x"] == "mx4" else st.x.double()
        if st.gain is not None:
            x = x / torch.sqrt((x ** 2).sum(-1, keepdim=True) / c["k"] + EPS) * st.gain.double()
        return torch.cat([x @ _exact_values(st.w[p:p + 256 * PANEL * -(-c["k"] // 128)], 16384, c["k"]).t()
                          for p in range(0, st.w.numel(), 256 * PANEL * -(-c["k"] // 128))], 1)[:, :c["n"]]
    z = st.z.double().cpu().numpy()
    bias = None if st.bias is None else st.bias.double().cpu().numpy()
    tokens, begin, end = (None if t is None else t.cpu().numpy() for t in (st.tokens, st.begin, st.end))
    allowed, mask_row = (None if t is None else t.cpu().numpy() for t in (st.allowed, st.mask_row))
    for r in range(c["rows"]):
        if tokens is not None:
            n = np.bincount(tokens[begin[r]:end[r]], minlength=c["vocab"])
            hit = n > 0
            pos = hit & (z[r] > 0)
            z[r][pos] /= st.repetition
            z[r][hit & ~pos] *= st.repetition
            z[r] -= st.frequency * n + st.presence * hit
        if bias is not None:
            z[r] += bias
        if allowed is not None:
            ok = np.unpackbits(allowed[mask_row[r]].view(np.uint8), bitorder="little")[:c["vocab"]]
            z[r][ok == 0] = -np.inf
    return z
