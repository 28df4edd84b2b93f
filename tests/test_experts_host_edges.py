"""Expert layers, host side: what the Python layer does before a launch, checked on the CPU with stand-ins for the device's calls."""
import threading

import pytest
import torch

from paper_2608_00358_b200 import binding as hb
from paper_2608_00358_b200 import experts as ex


@pytest.fixture
def no_device(monkeypatch):
    """Device memory from the host's, one stream, nothing captured."""
    real = torch.empty
    monkeypatch.setattr(ex.torch, "empty", lambda *a, **kw: real(*a, **{k: v for k, v in kw.items() if k != "device"}))
    monkeypatch.setattr(ex, "_stream", lambda dev: 7)
    monkeypatch.setattr(ex, "_capturing", lambda: False)


def test_scratch_is_not_shared_by_host_threads(no_device):
    """Calls of two launches may interleave between threads on one stream (the library is called without the interpreter's lock): what one thread's first launch
    left for its second must not be another's to write."""
    scratch = ex._Scratch()
    mine = scratch.get(0, 1000)
    seen = []
    t = threading.Thread(target=lambda: seen.append(scratch.get(0, 1000)))
    t.start()
    t.join()
    assert seen[0][1] != mine[1]
    assert scratch.get(0, 500)[1] == mine[1]  # the same thread and stream: the same memory
    assert scratch.get(0, 2000)[0].numel() >= 2000
