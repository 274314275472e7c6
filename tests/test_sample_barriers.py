"""Barriers of the sampling kernel that no run shows to be missing (a run without them goes wrong once in a great many), read
from its source."""
import os
import re

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_05650_b200", "csrc", "sample.cu")


def code():
    return re.sub(r"//[^\n]*|/\*.*?\*/", "", open(SOURCE).read(), flags=re.S)


def test_words_of_the_warps_are_read_before_they_are_written_again():
    """tokens_between reads the words that the next gather writes before its first barrier."""
    body = re.search(r"auto tokens_between = .*?\n            \};", code(), flags=re.S).group(0)
    last_read = body.rindex("s.warp_val[1][w]")
    assert "__syncthreads();" in body[last_read:body.rindex("return n;")]


def test_no_store_to_a_cta_that_may_not_run_yet():
    """All CTAs of a cluster arrive before they read anything, and wait before the first exchange."""
    kernel = code()
    kernel = kernel[kernel.index("sample_kernel(const SampleParams p)"):kernel.index("size_t sample_smem_bytes")]
    first = min(kernel.index(f) for f in ("gather<", "st_peer(", "put_candidate(", "share_bins(") if f in kernel)
    assert 0 < kernel.index("cluster_here();") < kernel.index("cluster_all_here();") < first
    assert kernel.count("cluster_here();") == kernel.count("cluster_all_here();") == 1
    assert "return" not in kernel[:first].replace("return x + 0.f;", "")        # (all threads get there)
