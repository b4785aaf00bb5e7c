"""A grammar of more states than a launch has workgroups."""
import numpy as np
import pytest

import synth
from test_gpu_head_rules import _shape, _weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [65535, 65537, 2 ** 24 + 1])
def test_many_masks(n):
    """The last state allows one token, the one before it nothing (and so masks nothing), the first one the other token; each token
    leads to the last state, then to the one before."""
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2602_05499_amd as P
    s = _shape("f32", 2)
    mask = synth.gen_skip_mask(s)
    ses = P.Session(s, _weights(s, mask), mask, max_seq=64, max_k=4)
    free = ses.generate(np.array([0, 1, 1], np.int32), 12, 3)[0]
    for tok in (0, 1):
        allowed = torch.zeros(n, 1, dtype=torch.int32, device="cuda")
        allowed[n - 1], allowed[0], allowed[n - 2] = 1 << tok, 2 >> tok, -4        # (bits past the vocabulary count for nothing)
        nxt = torch.full((n, 2), n - 1, dtype=torch.int32, device="cuda")
        for state, want in ((n - 1, [tok] * 12), (0, [1 - tok] + [tok] * 11)):
            ses.set_rules(allowed=allowed, next=nxt, state=state)
            for K in (0, 3):
                assert ses.generate(np.array([0, 1, 1], np.int32), 12, K)[0].tolist() == want
        nxt.fill_(n - 2)
        ses.set_rules(allowed=allowed, next=nxt, state=n - 2)
        assert np.array_equal(ses.generate(np.array([0, 1, 1], np.int32), 12, 3)[0], free)
    ses.close()
