"""Prompts whose waits run out: the kernel ends by itself, after its MMAs.  The order of that end is
read from the source; no result shows it."""
import os
import re

import paper_2606_12487_gb300


def _kernel():
    with open(os.path.join(os.path.dirname(paper_2606_12487_gb300.__file__), "csrc", "kv8_prefill.cu")) as f:
        src = re.sub(r"//[^\n]*", "", f.read())
    return src[src.index("kv8_prefill_kernel("):src.index("kv8_join_kernel(")]


def test_tensor_memory_is_freed_after_the_mmas_whoever_gave_up():
    k = _kernel()
    issue = k[k.index("const bool leader = elect_one();"):]
    # every path of the issuing warp commits, and both CTAs' MMA warps wait, with the full bound
    assert len(re.findall(r"commit\(&S\.drain\)", k)) == 1 and "if (!ok)" not in issue[:issue.index("__syncthreads")]
    assert issue.index("commit(&S.drain)") < issue.index("mbar_wait_warp(&S.drain") < issue.index("tmem_dealloc")
    assert "mbar_wait_warp(&S.drain, 0, &no_abort, c.err, kDevTimeoutDrain);" in issue
    assert "if (warp == kMmaWarp && nt > 0) {" in issue
