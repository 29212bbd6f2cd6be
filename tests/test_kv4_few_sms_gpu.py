"""Attention over the 4-bit cache where the library uses few SMs (DPTQ_MAX_GRID): one CTA, or one pair, at a time, so that no task
is cut along its keys."""
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
    sys.path.insert(0, "tests")
    import numpy as np
    import kv4_reference as ref
    from paper_2606_12487_gb300 import dptq
    from test_kv4_gpu import _check, _rows
    dptq.load()
    # few rows; prompts alone, of heads of 64 and 128, up to three tasks; pairs, one and three
    for ns, lens, H, g, D in (([1, 1], [3000, 40], 2, 4, 128), ([100], [2700], 1, 2, 64), ([100], [2700], 3, 2, 128),
                              ([40], [2600], 2, 1, 128), ([260], [2700], 1, 2, 128), ([260], [2900], 3, 2, 128),
                              ([40, 30], [2700, 90], 2, 1, 64)):
        rng = np.random.default_rng(H)
        cu, lens, table, blocks = ref.random_batch(rng, ns, lens, 16)
        _check(dptq, ref.random_cache(rng, blocks, H, 16, D), _rows(rng, sum(ns), H * g, D), cu, lens, table)
    print("all served")
""")


@pytest.mark.parametrize("sms", [1, 2, 3, 5])
def test_few_sms(sms):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    r = subprocess.run([sys.executable, "-c", CODE], cwd=ROOT, env=dict(os.environ, DPTQ_MAX_GRID=str(sms)), capture_output=True,
                       text=True, timeout=300)
    assert r.returncode == 0 and "all served" in r.stdout, r.stdout + r.stderr
