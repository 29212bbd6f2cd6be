"""What orders the stores of a prompt's second CTA before the MMAs that the first one issues, and the
scales of a tile before the softmax that reads them: the kernel's source is read, since a
missing order shows in no result that could be waited for."""
import os
import re

import paper_2606_12487_gb300

CSRC = os.path.join(os.path.dirname(paper_2606_12487_gb300.__file__), "csrc")


def _source(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def _function(src, name):
    at = src.index(name + "(")
    return src[at:src.index("\n}", at)]


def test_the_cluster_forms_release_and_acquire_at_cluster_scope():
    src = _source("dptq_device.cuh")
    assert "mbarrier.arrive.release.cluster.shared::cluster.b64" in _function(src, "void mbar_arrive_remote_release")
    assert "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64" in _function(src, "bool mbar_try_wait_cluster")


def test_only_tensor_memory_goes_by_the_unscoped_arrival():
    src = _source("kv8_prefill.cu")
    unscoped = [m.start() for m in re.finditer(r"\bmbar_arrive_remote\(", src)]
    assert len(unscoped) == 1
    lines = src[:unscoped[0]].rstrip().splitlines()
    assert lines[-2].strip().endswith("mbar_arrive_remote_release(cluster_map(smem_u32(bar), 0));")   # else if (stored)
    calls = re.findall(r"tell_first\((&S\.\w+)[^;]*, (true|false)\);", src)
    assert calls and all(stored == "true" or bar == "&S.pfull" for bar, stored in calls)
    assert ("&S.qfull", "true") in calls


def test_widened_tiles_and_queries_are_acquired_at_cluster_scope():
    src = _source("kv8_prefill.cu")
    issue = src[src.index("constexpr uint32_t kIdS"):]
    for bar in ("kfull", "vfull", "qfull"):
        waits = re.findall(r"(\w+)\(&S\.%s\[" % bar, issue[:issue.index("mma_s(t, s1);")])
        assert waits and set(waits) == {"wait_stored"}, bar
    assert re.search(r"wait_stored = [^;]*PAIR \? mbar_wait_near_cluster\(bar", issue)


def test_scales_are_waited_for_where_they_are_read():
    src = _source("kv8_prefill.cu")
    softmax = src[src.index("reg_more<160>"):src.index("reg_less<112>")]
    assert 0 < softmax.index("(&S.mfull[j % kMeta]") < softmax.index("= S.meta[")
    widen = src[src.index("reg_less<112>"):]
    assert widen.index("S.meta[j % kMeta][lane] =") < widen.index("mbar_arrive(&S.mfull[j % kMeta]);")
