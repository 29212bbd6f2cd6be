"""Prompts over the 4-bit cache whose waits run out: the kernel ends by itself, after its MMAs, and says so; and what orders the
stores of a pair's second CTA.  Orders are read from the source; no result shows them."""
import os
import re
import subprocess
import sys
import textwrap

import pytest

import paper_2606_12487_gb300

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _source():
    with open(os.path.join(os.path.dirname(paper_2606_12487_gb300.__file__), "csrc", "kv4_prefill.cu")) as f:
        src = re.sub(r"//[^\n]*", "", f.read())
    return src[:src.index("kv4_join_kernel(")]


def test_tensor_memory_is_freed_after_the_mmas_whoever_gave_up():
    k = _source()[_source().index("kv4_prefill_kernel("):]
    issue = k[k.index("const bool leader = elect_one();"):]
    assert len(re.findall(r"commit\(&S\.drain\)", k)) == 1 and "if (!ok)" not in issue[:issue.index("__syncthreads")]
    assert issue.index("commit(&S.drain)") < issue.index("mbar_wait_warp(&S.drain") < issue.index("tmem_dealloc")
    assert "mbar_wait_warp(&S.drain, 0, &no_abort, c.err, kDevTimeoutDrain);" in issue
    assert "if (warp == kMmaWarp && nt > 0) {" in issue


def test_waits_are_bounded_by_the_clock():
    src = _source()
    wait = src[src.index("bool wait_bounded("):src.index("bool wait_one(")]
    assert "clock64()" in wait and "now - t0 > limit" in wait


def test_a_pairs_stores_are_released_and_acquired_at_cluster_scope():
    src = _source()
    unscoped = [m.start() for m in re.finditer(r"\bmbar_arrive_remote\(", src)]
    assert len(unscoped) == 1
    lines = src[:unscoped[0]].rstrip().splitlines()
    assert lines[-2].strip().endswith("mbar_arrive_remote_release(cluster_map(smem_u32(bar), 0));")
    calls = re.findall(r"tell_first\((&S\.\w+)[^;]*, (true|false)\);", src)
    assert ("&S.qfull", "true") in calls and all(stored == "true" or bar == "&S.pfull" for bar, stored in calls)
    issue = src[src.index("constexpr uint32_t kIdS"):]
    for bar in ("kfull", "vfull", "qfull"):
        waits = re.findall(r"(\w+)\(&S\.%s\[" % bar, issue[:issue.index("mma_s(t, s1);")])
        assert waits and set(waits) == {"wait_stored"}, bar
    assert re.search(r"wait_stored = [^;]*PAIR \? wait_cluster\(bar", issue)
    softmax = src[src.index("reg_more<160>"):src.index("reg_less<112>")]
    assert 0 < softmax.index("(&S.mfull[j % kMeta]") < softmax.index("= S.gone[")
    widen = src[src.index("reg_less<112>"):]
    assert widen.index("S.gone[j % kMeta] =") < widen.index("mbar_arrive(&S.mfull[j % kMeta]);")


CHILD = """
import numpy as np, sys, torch
sys.path.insert(0, "tests")
import kv4_reference as ref
from paper_2606_12487_gb300 import dptq
rng = np.random.default_rng(0)
def call(ns, lens, H, g, D):
    cu, lens, table, blocks = ref.random_batch(rng, ns, lens, 16)
    cache = ref.random_cache(rng, blocks, H, 16, D)
    kc, vc, cut, lt, tt = [torch.from_numpy(np.ascontiguousarray(a)).cuda() for a in (cache[0], cache[2], cu, lens, table)]
    ks, vs = [torch.from_numpy(b.astype(np.int32)).to(torch.int16).cuda().view(torch.bfloat16) for b in (cache[1], cache[3])]
    c = dptq.Kv4Cache(kc, vc, ks, vs)
    b = dptq.Kv8Batch(cut, lt, tt, tokens=int(cu[-1]), max_tokens=max(ns), max_len=int(lens.max()))
    q = torch.from_numpy(rng.standard_normal((int(cu[-1]), H * g, D)).astype(np.float16)).cuda()
    out = torch.zeros_like(q)
    dptq.dptq_kv4_attention(c, b, q, out, 0.1)
    torch.cuda.synchronize()
    return out.cpu().numpy(), ref.attend(cache, q.cpu().numpy(), cu, lens, table, 0.1)

def right(out, want_tol):
    return bool((np.abs(out - want_tol[0]) <= want_tol[1]).all())
# alone, heads of 64; alone; cut along the keys; pairs; pairs cut along the keys
for ns, lens, H, g, D in (([300], [900], 80, 2, 64), ([130] * 20, [500] * 20, 8, 1, 128), ([200], [3000], 2, 1, 128),
                          ([600], [2700], 20, 2, 128), ([600], [3500], 2, 1, 128)):
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
    env = dict(os.environ, DPTQ_WAIT_CYCLES="200000", DPTQ_TEST_KV8_SHORTFALL=("%d0" % what) * 5)
    r = subprocess.run([sys.executable, "-c", textwrap.dedent(CHILD)], cwd=ROOT, env=env, capture_output=True, text=True,
                       timeout=300)
    assert r.returncode == 0 and "gave up and went on" in r.stdout, r.stdout + r.stderr
