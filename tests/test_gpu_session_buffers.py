"""What a session lets go of: rules and draft heads that later ones replaced are kept while the stream may still read them, and no
longer."""
import numpy as np
import pytest

import synth
from test_gpu_head_rules import _rule_sets, _shape, _weights

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2602_05499_amd as P
    return P


WAITS = {
    "generate": lambda s, p: s.generate(p, 6, 2),
    "read": lambda s, p: s.read(),
    "committed": lambda s, p: s.committed(),
    "prefill": lambda s, p: s.prefill(p),
    "dump_draft": lambda s, p: s.dump_draft(0),
    "sync": lambda s, p: s.sync(),
}


@pytest.mark.parametrize("which", list(WAITS))
def test_replaced_tensors_are_let_go(P, which):
    """A grammar and a head for every request, as many as there are requests: the memory stays that of one of them."""
    import gc
    import torch
    s = _shape("bf16", 2050)
    dw = _weights(s, synth.gen_skip_mask(s))
    prompt = synth.gen_prompt(3, 9, s.vocab)
    dev, _ = _rule_sets(s.vocab, np.random.default_rng(5))["all"]
    ses = P.Session(s, dw, synth.gen_skip_mask(s), max_seq=96, max_k=4)
    ses.prefill(prompt)
    held = []
    gc.collect()                                         # what earlier tests left behind
    for i in range(7):
        ses.set_rules(**{k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in dev.items()})
        ses.set_draft_head(P.mx4_quantize(dw.lm_head))
        ses.decode()
        WAITS[which](ses, prompt)
        held.append(torch.cuda.memory_allocated())
    assert len(set(held[2:])) == 1, held
    ses.close()
