"""Sources that only the block operators use are named block_*: the digest that
the rounds' stored counters go by leaves those out."""
import os
import re

import bench


def test_other_sources_belong_to_the_rounds():
    d = bench.KERNEL_SOURCES
    files = {f: open(os.path.join(d, f)).read() for f in os.listdir(d)}
    reached, todo = set(), [f for f in files if f.endswith((".hip", ".cpp")) and not f.startswith("block_")]
    while todo:
        f = todo.pop()
        if f not in reached:
            reached.add(f)
            todo += [h for h in re.findall(r'#include "([^"]+)"', files[f]) if h in files]
    assert reached == {f for f in files if not f.startswith("block_")}
