"""Prompts whose waits run out: the kernel ends by itself, after its MMAs, and says so.  The order of that
end and what bounds a wait are read from the source; no result shows them."""
import os
import re
import subprocess
import sys
import textwrap

import pytest

import paper_2606_12487_gb300

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _kernel():
    with open(os.path.join(os.path.dirname(paper_2606_12487_gb300.__file__), "csrc", "kv8_prefill.cu")) as f:
        src = re.sub(r"//[^\n]*", "", f.read())
    return src[:src.index("kv8_join_kernel(")]


def test_tensor_memory_is_freed_after_the_mmas_whoever_gave_up():
    k = _kernel()[_kernel().index("kv8_prefill_kernel("):]
    issue = k[k.index("const bool leader = elect_one();"):]
    # every path of the issuing warp commits, and both CTAs' MMA warps wait, with the full bound
    assert len(re.findall(r"commit\(&S\.drain\)", k)) == 1 and "if (!ok)" not in issue[:issue.index("__syncthreads")]
    assert issue.index("commit(&S.drain)") < issue.index("mbar_wait_warp(&S.drain") < issue.index("tmem_dealloc")
    assert "mbar_wait_warp(&S.drain, 0, &no_abort, c.err, kDevTimeoutDrain);" in issue
    assert "if (warp == kMmaWarp && nt > 0) {" in issue


def test_waits_are_bounded_by_the_clock():
    """A poll (try_wait) may be suspended for any time, so a number of polls bounds no wait."""
    src = _kernel()
    wait = src[src.index("bool wait_near("):src.index("bool mbar_wait_near(")]
    assert "clock64()" in wait and "now - t0 > limit" in wait and "polls" not in wait


CHILD = """
import numpy as np, sys, torch
sys.path.insert(0, "tests")
import kv8_reference as ref
from paper_2606_12487_gb300 import dptq
rng = np.random.default_rng(0)
def call(ns, lens, H, g, D):
    cu, lens, table, blocks = ref.random_batch(rng, ns, lens, 16)
    cache = ref.random_cache(rng, blocks, H, 16, D)
    kc, ks, vc, vs, cut, lt, tt = [torch.from_numpy(np.ascontiguousarray(a)).cuda() for a in (*cache, cu, lens, table)]
    c = dptq.Kv8Cache(kc, vc, ks, vs)
    b = dptq.Kv8Batch(cut, lt, tt, tokens=int(cu[-1]), max_tokens=max(ns), max_len=int(lens.max()))
    q = torch.from_numpy(rng.standard_normal((int(cu[-1]), H * g, D)).astype(np.float16)).cuda()
    out = torch.zeros_like(q)
    dptq.dptq_kv8_attention(c, b, q, out, 0.1)
    torch.cuda.synchronize()
    return out.cpu().numpy(), ref.attend(cache, q.cpu().numpy(), cu, lens, table, 0.1)

def right(out, want_tol):
    return bool((np.abs(out - want_tol[0]) <= want_tol[1]).all())
# alone, heads of 64; alone; split along the keys; pairs
for ns, lens, H, g, D in (([300], [900], 80, 2, 64), ([130] * 20, [500] * 20, 8, 1, 128), ([200], [3000], 2, 1, 128),
                          ([600, 520], [2000, 520], 16, 2, 128)):
    call(ns, lens, H, g, D)
    try:
        dptq.dptq_last_device_error()
        raise SystemExit("no wait ran out")
    except dptq.DptqError as e:
        assert e.status == 5 and "timed out" in str(e), e
    assert right(*call(ns, lens, H, g, D))
    dptq.dptq_last_device_error()
print("gave up and went on")
"""


@pytest.mark.gpu
@pytest.mark.parametrize("what", [1, 2, 3])     # the barrier that waits for one arrival more than there is
def test_a_wait_that_runs_out_ends_the_kernel(what):
    """DPTQ_TEST_KV8_SHORTFALL (a host-side hook): a barrier of every other call expects one arrival too
    many, in the CTAs of each form of the kernel.  The waits behind it end by their bound (0.1 ms), the
    call is reported as timed out, and the next one is right.  No fault is involved."""
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    env = dict(os.environ, DPTQ_WAIT_CYCLES="200000", DPTQ_TEST_KV8_SHORTFALL=("%d0" % what) * 4)
    r = subprocess.run([sys.executable, "-c", textwrap.dedent(CHILD)], cwd=ROOT, env=env, capture_output=True, text=True,
                       timeout=300)
    assert r.returncode == 0 and "gave up and went on" in r.stdout, r.stdout + r.stderr


BOTH = """
import numpy as np, torch
from paper_2606_12487_gb300 import dptq, inputs
W = torch.from_numpy(inputs.weights(4096, 4096, layer=1)).cuda()
x = torch.from_numpy(inputs.activations(inputs.llama2_7b_decode(), 32, 4096)).cuda()
layer = dptq.dptq_pack_weights(W, 4096)
y = torch.empty((32, 4096), dtype=torch.float16, device="cuda")
cache = dptq.Kv8Cache.empty(4, 1, 16, 128)
i32 = dict(dtype=torch.int32, device="cuda")
def attend(n, page):
    b = dptq.Kv8Batch(torch.tensor([0, n], **i32), torch.tensor([n], **i32), torch.full((1, 3), page, **i32),
                      tokens=n, max_tokens=n, max_len=n)
    q = torch.zeros((n, 1, 128), dtype=torch.float16, device="cuda")
    dptq.dptq_kv8_attention(cache, b, q, q.clone(), 0.1)
def answers(calls=3):
    got = []
    for _ in range(calls):
        try:
            dptq.dptq_last_device_error()
            got.append(0)
        except dptq.DptqError as e:
            got.append(e.status)
    return got
attend(1, 9)                               # a bad page, then a prompt that gives up
attend(33, 0)
print(answers())
attend(33, 9)                              # a bad page alone
print(answers())
attend(1, 9)                               # a bad page, then a GEMM that gives up
dptq.dptq_qlinear(layer, x, 4, y)
print(answers())
attend(1, 9)
ref = y.clone()
dptq.dptq_qlinear(layer, x, 4, ref)        # (their order does not matter, and the GEMM's scratch is clean)
print(answers(2))
dptq.dptq_qlinear(layer, x, 4, y)
print(answers(1), torch.equal(ref, y))
"""


@pytest.mark.gpu
def test_a_bad_page_hides_no_wait_that_gave_up():
    """Both are reported: first the time-out, whose call left its output incomplete, then the page."""
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    env = dict(os.environ, DPTQ_WAIT_CYCLES="200000", DPTQ_TEST_KV8_SHORTFALL="01", DPTQ_TEST_ROWS_SHORTFALL="1")
    r = subprocess.run([sys.executable, "-c", textwrap.dedent(BOTH)], cwd=ROOT, env=env, capture_output=True, text=True,
                       timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
    assert r.stdout.split("\n")[:5] == ["[5, 1, 0]", "[1, 0, 0]", "[5, 1, 0]", "[1, 0]", "[0] True"], r.stdout
