"""A KV8 call that would have to allocate its scratch is refused during stream capture, and works in a
capture after dptq_kv8_reserve (each in a fresh process)."""
import os
import subprocess
import sys
import textwrap

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CODE = textwrap.dedent("""
    import sys
    import torch
    from paper_2606_12487_gb300 import dptq
    dptq.load()
    c = dptq.Kv8Cache.empty(4, 2, 16, 64)
    i32 = dict(dtype=torch.int32, device="cuda")
    b = dptq.Kv8Batch(torch.tensor([0, 1], **i32), torch.tensor([20], **i32), torch.tensor([[2, 0]], **i32), tokens=1,
                      max_tokens=1, max_len=32)
    q, out = torch.zeros((1, 4, 64), device="cuda").half(), torch.ones((1, 4, 64), device="cuda").half()
    k = torch.ones((1, 2, 64), device="cuda").half()
    if sys.argv[1] == "reserve":
        dptq.dptq_kv8_reserve()
    torch.cuda.synchronize()
    g, status = torch.cuda.CUDAGraph(), []
    with torch.cuda.graph(g):
        out.mul_(2)
        for call in (lambda: dptq.dptq_kv8_append(c, b, k, k), lambda: dptq.dptq_kv8_attention(c, b, q, out, 0.1)):
            try:
                call()
                status.append(0)
            except dptq.DptqError as e:
                status.append(e.status)
    g.replay()
    torch.cuda.synchronize()
    print("status", status, out.float().mean().item())
""")


@pytest.mark.parametrize("what,want", [("none", "status [2, 2] 2.0"), ("reserve", "status [0, 0] 0.05")])
def test_capture(what, want):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    r = subprocess.run([sys.executable, "-c", CODE, what], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
    # one key in twenty is not zero: v = 1 at position 19, equal weights
    assert r.stdout.startswith(want[:len("status [2, 2] ")]), r.stdout
    assert abs(float(r.stdout.split()[-1]) - float(want.split()[-1])) < 1e-3
