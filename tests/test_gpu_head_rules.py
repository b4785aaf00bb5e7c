"""The draft's MXFP4 output head and the rules on logits inside a decode context: against the oracle's selection rules, against
the same model without them, and together, as a speculative program uses them."""
import numpy as np
import pytest

import synth
from test_gpu_mx4 import quantize64, values64
from test_gpu_rules import rules64
from test_gpu_select import _accept_off_boundary, _off_boundary

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2602_05499_amd as P
    return P


def _shape(dtype="f32", vocab=1100, **over):
    kw = dict(name="head_rules", n_layers=3, d_model=128, n_heads=4, n_kv_heads=2, head_dim=32, d_ffn=160, vocab=vocab, dtype=dtype,
              init_std=0.3, gain_std=0.1, n_skip=1, skip_layers=(1,), K=4)
    kw.update(over)
    return synth.CONFIGS["tiny"].with_(**kw)


def _weights(s, mask):
    from synth.device import DeviceWeights
    return DeviceWeights(s, damp_skipped=0.1, skip_mask=mask)


def _automaton(vocab, rng, n_states=5):
    """A grammar: about a third of the tokens allowed in each state, successors at random, some of them the free state."""
    ok = rng.random((n_states, vocab)) < 0.3
    ok[:, 7] = True
    nxt = rng.integers(0, n_states, (n_states, vocab)).astype(np.int32)
    nxt[rng.random((n_states, vocab)) < 0.02] = -1
    words = -(-vocab // 32)
    bits = np.zeros((n_states, words * 32), bool)
    bits[:, :vocab] = ok
    bits[:, vocab:] = True                               # bits past the vocabulary count for nothing
    allowed = np.packbits(bits, axis=1, bitorder="little").view(np.int32)
    return ok, nxt, allowed


class HostRules:
    """The rules of a context on the host: history, state, and a row's logits in float64."""

    def __init__(self, vocab, rep=1.0, pres=0.0, freq=0.0, bias=None, ok=None, nxt=None, state=0):
        self.kw = dict(rep=float(np.float32(rep)), pres=float(np.float32(pres)), freq=float(np.float32(freq)), bias=bias)
        self.vocab, self.ok, self.nxt, self.state, self.history = vocab, ok, nxt, state if ok is not None else -1, []

    def step(self, s, tok):
        if s < 0 or self.nxt is None:
            return s
        n = int(self.nxt[s, tok])
        return n if 0 <= n < len(self.ok) else -1

    def row(self, z, extra=()):
        """(logits, magnitudes) of the row behind the draft tokens `extra`."""
        h = np.array(list(self.history) + [int(t) for t in extra], np.int64)
        out, mag = rules64(z[None], h, [0], [len(h)], self.kw["rep"], self.kw["pres"], self.kw["freq"], self.kw["bias"], None, None)
        s = self.state
        for t in extra:
            s = self.step(s, int(t))
        if s >= 0 and self.ok[s].any():
            out[0, ~self.ok[s]] = -np.inf
        return out[0], mag[0]

    def commit(self, toks):
        for t in toks:
            self.history.append(int(t))
            self.state = self.step(self.state, int(t))


def _same(got, want, mag):
    fin = np.isfinite(want)
    assert np.array_equal(got[~fin], want[~fin].astype(np.float32))
    assert (np.abs(got[fin] - want[fin]) <= 6 * 2.0 ** -24 * mag[fin]).all()      # six float32 operations


def _rule_sets(vocab, rng):
    import torch
    bias = np.where(rng.random(vocab) < 0.2, 2 * rng.standard_normal(vocab), 0).astype(np.float32)
    ok, nxt, allowed = _automaton(vocab, rng)
    one = allowed[:1]
    t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()                 # noqa: E731
    pen = dict(repetition=1.3, presence=0.4, frequency=0.2)
    return {"penalties": (pen, dict(rep=1.3, pres=0.4, freq=0.2)),
            "bias and mask": (dict(bias=t(bias), allowed=t(one)), dict(bias=bias, ok=ok[:1])),
            "grammar": (dict(allowed=t(allowed), next=t(nxt), state=2), dict(ok=ok, nxt=nxt, state=2)),
            "all": (dict(bias=t(bias), allowed=t(allowed), next=t(nxt), state=0, **pen),
                    dict(bias=bias, ok=ok, nxt=nxt, rep=1.3, pres=0.4, freq=0.2))}


@pytest.mark.parametrize("dtype,vocab,n_prompt", [("f32", 1100, 9), ("bf16", 2050, 3), ("bf16", 1031, 40)])
@pytest.mark.parametrize("which", ["penalties", "bias and mask", "grammar", "all"])
def test_greedy_tokens_under_rules(P, dtype, vocab, n_prompt, which):
    """Plain decoding under rules against the same model without them, whose raw logits go through the host's rules and whose
    next token is the one the rules leave; then speculation: the same tokens, every draft and verify row under its own history."""
    s = _shape(dtype, vocab)
    mask = synth.gen_skip_mask(s)
    dw = _weights(s, mask)
    rng = np.random.default_rng(vocab + n_prompt)
    dev, host = _rule_sets(vocab, rng)[which]
    prompt = synth.gen_prompt(3, n_prompt, vocab)
    G, K = 24, s.K
    raw, ses = (P.Session(s, dw, mask, max_seq=128, max_k=K) for _ in range(2))
    raw.keep_logits(True)
    ses.keep_logits(True)
    ses.set_rules(**dev)
    hr = HostRules(vocab, **host)
    hr.commit([])
    hr.history += [int(t) for t in prompt]
    raw.prefill(prompt)
    ses.prefill(prompt)
    toks = []
    for i in range(G):
        want, mag = hr.row(raw.dump_logits(P.SD_LOGITS_VERIFY, 1)[0].astype(np.float64))
        got = ses.dump_logits(P.SD_LOGITS_VERIFY, 1)[0]
        _same(got, want, mag)
        tok = int(np.argmax(got))
        assert ses.read()[1]["t_last"] == tok
        toks.append(tok)
        hr.commit([tok])
        raw.set_pending(n_prompt + i, tok)
        raw.decode()
        ses.decode()
    ses.prefill(prompt)                                  # a new sequence: history and state start again
    hr = HostRules(vocab, **host)
    hr.history += [int(t) for t in prompt]
    hr.commit([ses.read()[1]["t_last"]])
    n_acc = 0
    while len(hr.history) - n_prompt < G:
        ses.draft(K)
        d = ses.dump_draft(K)
        ses.verify()
        zq, zp = ses.dump_logits(P.SD_LOGITS_DRAFT, K), ses.dump_logits(P.SD_LOGITS_VERIFY, K + 1)
        assert [int(t) for t in d] == [int(np.argmax(zq[i])) for i in range(K)]
        for z, n in ((zq, K), (zp, K + 1)):              # masked entries and nothing else are -inf
            for i in range(n):
                want, _ = hr.row(np.zeros(vocab), d[:i])
                assert np.array_equal(np.isneginf(z[i]), np.isneginf(want)), (i, n)
        ses.accept()
        ses.rollback()
        st = ses.read()[1]
        hr.commit(list(d[:st["last_n"]]) + [st["t_last"]])
        n_acc += st["last_n"]
    assert n_acc > 0
    assert [int(t) for t in hr.history[n_prompt:n_prompt + G]] == toks
    assert [int(t) for t in ses.read()[0][:G]] == toks
    raw.close()
    ses.close()


@pytest.mark.parametrize("which", ["penalties", "all"])
@pytest.mark.parametrize("mx4", [False, True])
def test_sampled_steps_under_rules(P, which, mx4):
    """Sampling: draws and accepts follow the oracle's rules on the processed rows, with lm_head and with the MXFP4 draft head."""
    from oracle import accept_sample, inv_cdf, softmax64
    s = _shape("f32", 1300)
    mask = synth.gen_skip_mask(s)
    dw = _weights(s, mask)
    dev, host = _rule_sets(s.vocab, np.random.default_rng(5))[which]
    K, T, n = 3, 0.8, 6
    ses = P.Session(s, dw, mask, max_seq=96, max_k=K, temperature=T)
    ses.set_rules(**dev)
    if mx4:
        ses.set_draft_head()
    prompt = synth.gen_prompt(3, 7, s.vocab)
    u = synth.gen_uniforms(78, 1 + n * (2 * K + 1))
    hr = HostRules(s.vocab, **host)
    hr.history += [int(t) for t in prompt]
    ses.prefill(prompt, P.SD_SAMPLE, u[:1])
    z = ses.dump_logits(P.SD_LOGITS_VERIFY, 1)[0]
    assert _off_boundary(softmax64(z, T), u[0]) and ses.read()[1]["t_last"] == inv_cdf(softmax64(z, T), u[0])
    hr.commit([ses.read()[1]["t_last"]])
    for i in range(n):
        us = u[1 + i * (2 * K + 1):1 + (i + 1) * (2 * K + 1)]
        ses.draft(K, P.SD_SAMPLE, us[:K])
        d, zq = ses.dump_draft(K), ses.dump_logits(P.SD_LOGITS_DRAFT, K)
        ses.verify()
        zp = ses.dump_logits(P.SD_LOGITS_VERIFY, K + 1)
        ses.accept(P.SD_SAMPLE, us[K:])
        ses.rollback()
        st = ses.read()[1]
        for j in range(K):
            assert np.array_equal(np.isneginf(zq[j]), np.isneginf(hr.row(np.zeros(s.vocab), d[:j])[0]))
            assert _off_boundary(softmax64(zq[j], T), us[j]) and int(d[j]) == inv_cdf(softmax64(zq[j], T), us[j])
        assert _accept_off_boundary(d, zq, zp, us[K:2 * K], float(us[2 * K]), T)
        assert (st["last_n"], st["t_last"]) == accept_sample(d, zq, zp, us[K:2 * K], float(us[2 * K]), T)
        hr.commit(list(d[:st["last_n"]]) + [st["t_last"]])
    ses.close()


@pytest.mark.parametrize("dtype,d,vocab", [("f32", 128, 1100), ("bf16", 256, 2049), ("bf16", 160, 65)])
def test_draft_head(P, dtype, d, vocab):
    """Draft rows end in the quantised head: their logits are those of a model whose lm_head holds the quantised values (same
    residual row, bit for bit; the two products differ by float32 rounding, at most (3 ceil(d / 32) + 16) 2^-23 of the sum of
    magnitudes each), verification and the output stay the target's, and the skip mask may change under it."""
    import torch
    s = _shape(dtype, vocab, d_model=d, n_heads=d // 32, n_kv_heads=d // 32)
    mask = synth.gen_skip_mask(s)
    dw = _weights(s, mask)
    K, G = 4, 20
    prompt = synth.gen_prompt(5, 11, vocab)
    head = P.mx4_quantize(dw.lm_head)
    code, e = quantize64(dw.lm_head.double().cpu().numpy())
    values = values64(code, e)
    ses = P.Session(s, dw, mask, max_seq=96, max_k=K)
    plain, _ = ses.generate(prompt, G, 0)
    ref_tokens, ref_stats = ses.generate(prompt, G, K)
    ses.keep_logits(True)
    ses.set_draft_head(head)
    got, stats = ses.generate(prompt, G, K)
    assert np.array_equal(got, plain) and np.array_equal(got, ref_tokens)
    # the same drafts from a model that has the quantised head for its own
    import copy
    dq = copy.copy(dw)
    dq.lm_head = torch.from_numpy(values).to(dw.lm_head.dtype).cuda()
    assert torch.equal(dq.lm_head.double().cpu(), torch.from_numpy(values))
    other = P.Session(s, dq, mask, max_seq=96, max_k=K)
    other.keep_logits(True)
    first = int(plain[0])
    for m in (mask, np.array([3, 0, 1], np.uint8)):
        for x in (ses, other):
            x.set_skip_mask(m)
            x.prefill(prompt)
            x.set_pending(len(prompt), first)
            x.draft(1)
        a, b = ses.dump_logits(P.SD_LOGITS_DRAFT, 1)[0], other.dump_logits(P.SD_LOGITS_DRAFT, 1)[0]
        # the normalised row has a mean square of 1 before its gain of at most 1.5: sum |x w| <= 1.5 sqrt(d) |w|_2
        tol = 2 * (3 * -(-d // 32) + 16) * 2.0 ** -23 * 1.5 * np.sqrt(d) * np.sqrt((values ** 2).sum(1))
        assert (np.abs(a - b) <= tol).all() and np.abs(a - b).max() > 0 or np.array_equal(a, b)
        assert int(ses.dump_draft(1)[0]) == int(np.argmax(a))
        for x in (ses, other):
            x.verify(); x.accept(); x.rollback()
    ses.set_skip_mask(np.full(3, 3, np.uint8))           # nothing left to run: the draft keeps lm_head
    ses.prefill(prompt)
    ses.draft(2)
    zq = ses.dump_logits(P.SD_LOGITS_DRAFT, 2)
    ses.verify(); ses.accept(); ses.rollback()
    ses.set_draft_head(False)
    ses.prefill(prompt)
    ses.draft(2)
    assert np.array_equal(zq, ses.dump_logits(P.SD_LOGITS_DRAFT, 2))
    ses.verify(); ses.accept(); ses.rollback()
    ses.set_skip_mask(mask)
    assert np.array_equal(ses.generate(prompt, G, K)[0], plain)
    ses.close()
    other.close()


def test_rules_set_on_a_running_sequence_and_taken_off(P):
    """Rules that come in the middle of a sequence count its prompt and tokens so far; without rules the tokens are as ever; a
    state that allows nothing masks nothing; between draft and rollback they cannot change."""
    import torch
    s = _shape("f32", 1100)
    mask = synth.gen_skip_mask(s)
    dw = _weights(s, mask)
    prompt = synth.gen_prompt(3, 9, s.vocab)
    ses = P.Session(s, dw, mask, max_seq=96, max_k=4)
    free, _ = ses.generate(prompt, 16, 4)
    ses.prefill(prompt)
    for _ in range(4):
        ses.decode()
    toks = ses.read()[0]
    assert np.array_equal(toks, free[:5])
    ses.set_rules(frequency=0.9, presence=0.2)
    hr = HostRules(s.vocab, freq=0.9, pres=0.2)
    hr.history += [int(t) for t in prompt] + [int(t) for t in toks]
    raw = P.Session(s, dw, mask, max_seq=96, max_k=4)
    raw.keep_logits(True)
    raw.prefill(np.concatenate([prompt, toks[:-1]]))
    raw.set_pending(len(prompt) + 4, int(toks[-1]))
    raw.decode()
    ses.decode()
    want, mag = hr.row(raw.dump_logits(P.SD_LOGITS_VERIFY, 1)[0].astype(np.float64))
    got = ses.dump_logits(P.SD_LOGITS_VERIFY, 1)[0]
    assert (np.abs(got - want) <= 6 * 2.0 ** -24 * mag + 1e-4).all()               # (the prompt went through other kernels)
    ses.draft(2)
    with pytest.raises(P.SdError) as e:
        ses.set_rules(presence=1.0)
    assert e.value.code == P.SD_ESTATE
    ses.verify(); ses.accept(); ses.rollback()
    ses.set_rules()
    assert np.array_equal(ses.generate(prompt, 16, 4)[0], free)
    ses.set_rules(allowed=torch.zeros(1, -(-s.vocab // 32), dtype=torch.int32, device="cuda"))
    assert np.array_equal(ses.generate(prompt, 16, 4)[0], free)
    ses.set_rules(bias=torch.full((s.vocab,), float("-inf"), device="cuda"))
    assert (ses.generate(prompt, 6, 2)[0] == 0).all()
    for bad in (dict(bias=torch.zeros(5, device="cuda")), dict(bias=torch.zeros(s.vocab)), dict(repetition=0.0),
                dict(next=torch.zeros(1, s.vocab, dtype=torch.int32, device="cuda"))):
        with pytest.raises(P.SdError) as e:
            ses.set_rules(**bad)
        assert e.value.code == P.SD_EINVAL
    with pytest.raises(P.SdError):
        ses.set_draft_head(P.mx4_quantize(dw.lm_head[:64]))
    ses.close()
    raw.close()


def test_tensors_still_in_the_making(P):
    """A head and rules whose tensors the current stream has yet to write, for a context on another stream; refused arguments
    leave what was set."""
    import torch
    s = _shape("bf16", 2050)
    mask = synth.gen_skip_mask(s)
    dw = _weights(s, mask)
    prompt = synth.gen_prompt(3, 21, s.vocab)
    dev, _ = _rule_sets(s.vocab, np.random.default_rng(5))["all"]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    ses = P.Session(s, dw, mask, max_seq=128, max_k=4, stream=stream)
    ses.set_draft_head(P.mx4_quantize(dw.lm_head))
    ses.set_rules(**dev)
    want, stats = ses.generate(prompt, 24, 4)
    torch.cuda.synchronize()
    big = torch.randn(4096, 4096, device="cuda")
    late = {k: torch.zeros_like(v) if isinstance(v, torch.Tensor) else v for k, v in dev.items()}
    head = P.Mx4(torch.zeros_like(ses.draft_head.data), s.vocab, s.d_model)
    torch.cuda.synchronize()
    for _ in range(20):
        big = (big @ big).clamp_(-1, 1)                      # what the writes below wait behind
    head.data.copy_(ses.draft_head.data)
    for k, v in late.items():
        if isinstance(v, torch.Tensor):
            v.copy_(dev[k])
    ses.set_draft_head(head)
    ses.set_rules(**late)
    got, again = ses.generate(prompt, 24, 4)
    assert np.array_equal(got, want) and again["accepted"] == stats["accepted"]
    one = dev["allowed"][:1]
    for bad in (dict(allowed=one[:0]), dict(allowed=5), dict(allowed=one, state=1), dict(allowed=one, state=2 ** 32), dict(allowed=one, state=-2)):
        with pytest.raises(P.SdError) as e:
            ses.set_rules(**bad)
        assert e.value.code == P.SD_EINVAL
    assert np.array_equal(ses.generate(prompt, 24, 4)[0], want)
    ses.close()


@pytest.mark.parametrize("vocab,K", [(1, 8), (1024, 8), (1025, 1), (300001, 8)])
def test_picks_around_the_chunks_of_a_row(P, vocab, K):
    """Greedy picks of draft and verify rows at vocabularies around the chunks that a row is cut into (1024 entries, longer ones
    past 262144), at the largest depth, on rows with equal entries and with none above -inf: the lowest index of the largest."""
    import torch
    s = _shape("f32", vocab, K=K, d_model=64, n_heads=2, n_kv_heads=2, n_layers=2, skip_layers=(1,))
    mask = synth.gen_skip_mask(s)
    dw = _weights(s, mask)
    dw.lm_head[vocab // 2:] = dw.lm_head[:vocab - vocab // 2].clone()             # every entry twice
    torch.cuda.synchronize()
    ses = P.Session(s, dw, mask, max_seq=64, max_k=K)
    if vocab > 1:
        ses.set_draft_head()
    ses.set_rules(frequency=0.01)
    ses.prefill(synth.gen_prompt(3, 5, vocab))
    for _ in range(3):
        ses.draft(K)
        d, zq = ses.dump_draft(K), ses.dump_logits(P.SD_LOGITS_DRAFT, K)
        ses.verify()
        zp = ses.dump_logits(P.SD_LOGITS_VERIFY, K + 1)
        ses.accept()
        ses.rollback()
        st = ses.read()[1]
        assert [int(t) for t in d] == [int(np.argmax(r)) for r in zq]
        n = 0
        while n < K and d[n] == np.argmax(zp[n]):
            n += 1
        assert (st["last_n"], st["t_last"]) == (n, int(np.argmax(zp[n])))
    ses.set_rules(bias=torch.full((vocab,), float("nan"), device="cuda"))
    ses.draft(K)
    assert (ses.dump_draft(K) == 0).all()
    ses.verify(); ses.accept(); ses.rollback()
    assert ses.read()[1]["last_n"] == K
    ses.close()


@pytest.mark.parametrize("mode", ["greedy", "sample"])
def test_everything_together_on_another_stream(P, mode):
    """A speculative program with the MXFP4 draft head, penalties and a grammar, on a stream of its own and in a static-workspace
    context: the grammar holds, greedy output equals plain decoding under the same rules, and both contexts agree."""
    import torch
    s = _shape("bf16", 2050)
    mask = synth.gen_skip_mask(s)
    dw = _weights(s, mask)
    rng = np.random.default_rng(11)
    dev, host = _rule_sets(s.vocab, rng)["all"]
    prompt = synth.gen_prompt(3, 21, s.vocab)
    K, G = 4, 30
    md = P.SD_SAMPLE if mode == "sample" else P.SD_GREEDY
    uni = synth.gen_uniforms(5, 1 + (2 * K + 1) * G)
    outs = []
    for static in (False, True):
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        ses = P.Session(s, dw, mask, max_seq=128, max_k=K, stream=stream, static_workspace=static)
        ses.set_draft_head()
        ses.set_rules(**dev)
        out, stats = ses.generate(prompt, G, K, md, uni)
        outs.append(out)
        ok, state = host["ok"], 0
        for t in out:
            assert state < 0 or ok[state, t]
            state = int(host["nxt"][state, t]) if state >= 0 else -1
        if mode == "greedy":
            assert np.array_equal(ses.generate(prompt, G, 0)[0], out)
        assert stats["accepted"] > 0
        ses.close()
    assert np.array_equal(outs[0], outs[1])
