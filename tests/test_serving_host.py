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


def test_workspace_lives_through_its_launch(monkeypatch):
    """A call on the same stream from another host thread, between this call's look-up of the workspace and its launch, may
    replace the workspace; the one that this call launches with stays."""
    import gc
    import threading
    import types
    import weakref

    import torch
    from paper_2608_12703_gb300 import serving

    made, alive = [], []
    zeros = torch.zeros

    def tracked(*a, **kw):
        x = zeros(*a, **kw)
        made.append((x.data_ptr(), weakref.ref(x)))
        return x

    monkeypatch.setattr(torch, "zeros", tracked)
    monkeypatch.setattr(serving, "_capturing", lambda: False)
    monkeypatch.setattr(serving, "_current_device", lambda: 0)
    monkeypatch.setattr(serving, "_raw_stream", lambda device: 7)
    monkeypatch.setattr(serving.PagedCache, "_rows", lambda self, q, *a: serving.A.AsrPagedRows())
    c = object.__new__(serving.PagedCache)
    c.device, c.dtype, c._index, c._ref, c._ws = torch.device("cpu"), torch.float32, 0, None, {}
    c._lock, c._attend_layouts = threading.Lock(), {}
    c._lib = types.SimpleNamespace(asr_spec_paged_attend_ws=lambda cache, rows: 64 * len(calls))
    calls = [0]
    n = zeros(1, dtype=torch.int32)

    def launch(cache, rows, out, lse, ws, size, stream):
        if len(calls) < 4:              # another thread's call comes first, and needs more
            calls.append(0)
            c.attend(zeros(1, len(calls), 2, 64), n)
            gc.collect()
        at = [ref for ptr, ref in made if ptr == ws and ref() is not None]
        alive.append(len(at) == 1 and at[0]().numel() >= size)
        return 0

    c._attend = launch
    c.attend(zeros(1, 1, 2, 64), n)
    assert alive == [True] * 4


@pytest.mark.parametrize("x", ["1", [1.0], None, 1j, 10 ** 400, b"2"], ids=lambda x: str(x)[:10])
def test_numbers_are_refused_with_the_package_error(x):
    from paper_2608_12703_gb300 import asrspec as A
    from paper_2608_12703_gb300 import serving
    with pytest.raises(A.AsrSpecError, match="ASR_E_INVAL scale"):
        serving._number(x, "scale")
    if not isinstance(x, int):
        with pytest.raises(A.AsrSpecError, match="ASR_E_INVAL budget"):
            serving._integer(x, "budget")
