"""CTAs of a cluster read one another's shared memory, and leave behind a barrier: a read that is still on its way when its owner has
left is undefined.  Whether it is cannot be seen from outside, so the sources are read: every barrier of a cluster orders memory."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "paper_2508_16201_b200", "csrc")


def test_every_cluster_barrier_orders_memory():
    found = {"arrive": 0, "wait": 0}
    for name in sorted(os.listdir(CSRC)):
        if not name.endswith((".cu", ".cuh", ".h")):
            continue
        with open(os.path.join(CSRC, name)) as f:
            text = re.sub(r"//[^\n]*", "", f.read())
        for half, how in re.findall(r"barrier\.cluster\.(arrive|wait)([a-z.]*)", text):
            assert {"arrive": ".release", "wait": ".acquire"}[half] in how, (name, half, how)
            found[half] += 1
    assert found["arrive"] > 0 and found["arrive"] == found["wait"]


def test_kernels_that_read_other_ctas_memory_end_with_a_barrier():
    """The last remote read of each kernel is followed by one."""
    for name in ("attn.cu", "attn_tc.cu", "accept.cu"):
        with open(os.path.join(CSRC, name)) as f:
            text = f.read()
        last = max(m.end() for m in re.finditer(r"ld_cluster_f32x?4?\(|ld\.shared::cluster|cluster_map\(", text))
        assert re.search(r"\bcluster_barrier\(\);", text[last:]), name
