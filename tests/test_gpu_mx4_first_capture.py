"""The product kernels' first calls of a process, inside a capture: what they set up once per device must not need an eager call."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

# rows and outputs of each tile kernel, and of the kernel for a few rows
SIZES = [("float32", 129, 11009), ("float32", 300, 11009), ("float32", 520, 11009), ("bfloat16", 100, 6001), ("bfloat16", 200, 11009),
         ("bfloat16", 520, 11009), ("mx4", 100, 8003), ("mx4", 1100, 7777), ("float32", 1, 8200), ("bfloat16", 7, 1003), ("mx4", 5, 8200)]


def child():
    import torch
    import paper_2602_05499_amd as P
    g = torch.Generator("cuda").manual_seed(1)
    k = 300
    ws = {n: P.mx4_quantize(torch.randn(n, k, device="cuda", generator=g)) for _, _, n in SIZES}
    xs = [torch.randn(m, k, device="cuda", generator=g).to(torch.bfloat16 if t == "bfloat16" else torch.float32) for t, m, _ in SIZES]

    def run():
        return [P.mx4_matmul(P.mx4_quantize(x) if t == "mx4" else x, ws[n]) for (t, m, n), x in zip(SIZES, xs)]

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ys = run()
    for _ in range(3):
        for x in xs:
            x.normal_(generator=g)
        graph.replay()
        torch.cuda.synchronize()
        for size, y, want in zip(SIZES, ys, run()):
            assert torch.equal(y, want), size
    print("captured first calls agree", flush=True)


def test_first_calls_of_a_process_inside_a_capture():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    here = os.path.dirname(os.path.abspath(__file__))
    env = dict(os.environ, PYTHONPATH=os.pathsep.join([os.path.dirname(here), here, os.environ.get("PYTHONPATH", "")]))
    r = subprocess.run([sys.executable, "-c", "import test_gpu_mx4_first_capture as t; t.child()"], env=env, capture_output=True, text=True,
                       timeout=100)
    assert r.returncode == 0 and "captured first calls agree" in r.stdout, r.stdout[-2000:] + r.stderr[-4000:]
