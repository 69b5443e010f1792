"""Rules of the programming model that a run on the device shows only by chance, checked in the kernels' text."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_21594_b200", "csrc")


def kernel(file, name):
    """The text of a kernel: from its name to the closing brace at the start of a line, without comments."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, file)).read())
    at = text.index(name + "(")
    return text[at:text.index("\n}\n", at)]


def test_blocks_meet_before_one_writes_into_the_others_shared_memory():
    """A block's shared memory may be touched by another block of its cluster only once it runs, which a meeting of the cluster shows."""
    body = kernel("layer_norm.cu", "norm_backward_kernel")
    first_store = body.index("row_sums<")                 # stores through map_shared_rank when the rows are cut between two blocks
    assert re.search(r"if constexpr \(CLUSTER > 1\) cg::this_cluster\(\)\.sync\(\);", body[:first_store])
    joined = body.index("map_shared_rank(joined")
    assert "cl.sync()" in body[body.index("if constexpr (JOIN > 1)"):joined]
