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
