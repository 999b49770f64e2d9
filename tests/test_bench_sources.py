"""The sources whose hash a measured traffic figure carries (no GPU needed)."""
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2405_18628_gb300", "csrc")


def test_the_hash_covers_what_the_attention_is_made_of():
    """The attention kernels, the entry points and every file of theirs that these include."""
    import bench
    seen, todo = set(), ["ppd_attention.cu", "ppd_attention_rows.cu", "ppd_api.cu"]
    while todo:
        name = todo.pop()
        if name in seen or not os.path.exists(os.path.join(CSRC, name)):
            continue
        seen.add(name)
        with open(os.path.join(CSRC, name)) as f:
            todo += re.findall(r'#include "([^"]+)"', f.read())
    assert set(bench.ATTENTION_SOURCES) == seen
