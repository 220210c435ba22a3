"""Host-side checks of the operators over a paged cache that need no GPU."""
import os
import re

import pytest

from paper_2608_12703_gb300 import build as B


def kernels():
    """Every kernel of the library that reaches into other blocks' shared memory: (file, name, body)."""
    for path in B.sources():
        with open(path) as f:
            text = re.sub(r"//[^\n]*", "", f.read())
        for m in re.finditer(r"__global__[^;{]*?\b((?!__launch_bounds__)\w+)\s*\([^;{]*?\)\s*\{", text):
            depth, at = 1, m.end()
            while depth:
                depth += {"{": 1, "}": -1}.get(text[at], 0)
                at += 1
            body = text[m.end():at]
            if re.search(r"\bdsmem_addr\(|\b(?:ld|st)_cluster\(", body):
                yield os.path.basename(path), m.group(1), body


@pytest.mark.parametrize("file,name,body", list(kernels()), ids=lambda x: x if len(x) < 60 else "")
def test_no_remote_shared_memory_before_the_cluster_has_started(file, name, body):
    """Shared memory of another block may be touched only once all blocks of the cluster are known to run: a barrier of the
    whole cluster comes first."""
    first = re.search(r"\bdsmem_addr\(|\b(?:ld|st)_cluster\(", body).start()
    barrier = re.search(r"\bcluster_(?:sync|wait)\(\)", body)
    assert barrier and barrier.start() < first
