"""The draft head and the rules in calls that the documentation allows and no ordinary program makes: vocabularies of one and two
tokens, blocks proposed from outside, a head that changes while its drafts are in flight."""
import numpy as np
import pytest

import synth
from test_gpu_head_rules import HostRules, _rule_sets, _same, _shape, _weights

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2602_05499_amd as P
    return P


@pytest.mark.parametrize("vocab", [1, 2, 3])
@pytest.mark.parametrize("mode", ["greedy", "sample"])
def test_smallest_vocabularies(P, vocab, mode):
    s = _shape("f32", vocab)
    mask = synth.gen_skip_mask(s)
    ses = P.Session(s, _weights(s, mask), mask, max_seq=64, max_k=4)
    prompt = np.zeros(5, np.int32)
    md, G, K = (P.SD_SAMPLE if mode == "sample" else P.SD_GREEDY), 12, 3
    u = synth.gen_uniforms(9, 1 + (2 * K + 1) * G)
    ses.set_rules(frequency=0.3, presence=0.1)
    plain = ses.generate(prompt, G, 0)[0]
    for head in (None, True):
        ses.set_draft_head(head)
        out, stats = ses.generate(prompt, G, K, md, u)
        assert ((0 <= out) & (out < vocab)).all()
        if mode == "greedy":
            assert np.array_equal(out, plain)
        if vocab == 1:
            assert stats["accepted"] == stats["drafted"] > 0
    ses.close()


@pytest.mark.parametrize("which", ["penalties", "grammar", "all"])
def test_proposed_blocks_under_rules(P, which):
    """sd_set_draft: every verify row goes through the rules under its own history, the proposed tokens in front of it included, and
    the state and counts go on from what was accepted."""
    s = _shape("f32", 1100)
    mask = synth.gen_skip_mask(s)
    dw = _weights(s, mask)
    rng = np.random.default_rng(4)
    dev, host = _rule_sets(s.vocab, rng)[which]
    prompt = synth.gen_prompt(3, 9, s.vocab)
    raw, ses = (P.Session(s, dw, mask, max_seq=96, max_k=4) for _ in range(2))
    raw.keep_logits(True)
    ses.set_rules(**dev)
    hr = HostRules(s.vocab, **host)
    hr.history += [int(t) for t in prompt]
    raw.prefill(prompt)
    ses.prefill(prompt)
    last, at = int(ses.read()[1]["t_last"]), len(prompt)
    hr.commit([last])
    for K in (4, 1, 0, 3):
        d = [int(t) for t in rng.integers(0, s.vocab, K)]
        if K == 3:                                       # a block that is accepted: what the model under its rules says itself
            probe = []
            for i in range(K):
                raw.set_pending(at, last)
                raw.set_draft(probe)
                raw.verify()
                probe.append(int(np.argmax(hr.row(raw.dump_logits(P.SD_LOGITS_VERIFY, i + 1)[i].astype(np.float64), probe)[0])))
                raw.accept(); raw.rollback()
            d = probe
        raw.set_pending(at, last)
        for x in (raw, ses):
            x.set_draft(d)
            x.verify()
        zr, zp = raw.dump_logits(P.SD_LOGITS_VERIFY, K + 1), ses.dump_logits(P.SD_LOGITS_VERIFY, K + 1)
        for i in range(K + 1):
            _same(zp[i], *hr.row(zr[i].astype(np.float64), d[:i]))
        for x in (raw, ses):
            x.accept()
            x.rollback()
        st = ses.read()[1]
        n = next((i for i in range(K) if d[i] != int(np.argmax(zp[i]))), K)
        assert (st["last_n"], st["t_last"]) == (n, int(np.argmax(zp[n])))
        assert K != 3 or n == 3
        hr.commit(d[:n] + [st["t_last"]])
        last, at = int(st["t_last"]), at + n + 1
    raw.close()
    ses.close()


def test_a_head_that_changes_behind_its_drafts(P):
    """Drafts in flight keep the head they were enqueued with; verification does not care."""
    s = _shape("bf16", 2050)
    mask = synth.gen_skip_mask(s)
    dw = _weights(s, mask)
    prompt = synth.gen_prompt(3, 9, s.vocab)
    ses = P.Session(s, dw, mask, max_seq=96, max_k=4)
    plain = ses.generate(prompt, 21, 0)[0]
    heads = [P.mx4_quantize(dw.lm_head), None, P.mx4_quantize(-dw.lm_head), True]
    ses.prefill(prompt)
    i = 0
    while ses.committed() < 21:
        ses.draft(4)
        ses.set_draft_head(heads[i % 4])
        ses.verify()
        ses.accept()
        ses.rollback()
        i += 1
    assert np.array_equal(ses.read()[0][:21], plain)
    ses.close()
