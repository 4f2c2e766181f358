"""The binding's default workspaces and host threads, on the host."""
import threading

import pytest
import torch

from paper_2606_08411_amd import _lib

CPU = torch.device("cpu")


@pytest.fixture
def not_capturing(monkeypatch):
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)


@pytest.mark.parametrize("kind", ["attn", "lmhead", "attn_kv4", "lmhead_mx4"])
def test_threads_on_one_stream_have_workspaces_of_their_own(not_capturing, kind):
    """A call is a kernel that writes partials and one that joins them, enqueued without the interpreter's
    lock: on a buffer in common, another thread's first kernel could come in between."""
    n = 4
    all_have_one, got = threading.Barrier(n), [None] * n

    def work(i):
        a, _ = _lib._workspace(kind, 1000, CPU, 7)
        all_have_one.wait()          # every thread is alive, as two threads inside a call are
        b, _ = _lib._workspace(kind, 500, CPU, 7)
        got[i] = (a.data_ptr(), b.data_ptr())
        all_have_one.wait()
    threads = [threading.Thread(target=work, args=(i,)) for i in range(n)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert all(a == b for a, b in got)          # a thread keeps its buffer
    assert len({a for a, _ in got}) == n


def test_workspaces_of_one_thread(not_capturing):
    """One per kind and stream; one that grows is at least doubled and the old one is not freed."""
    small, n = _lib._workspace("test", 1000, CPU, 1)
    assert n == small.numel() >= 1000
    assert _lib._workspace("test", 10, CPU, 1)[0] is small
    assert _lib._workspace("test", 10, CPU, 2)[0] is not small
    assert _lib._workspace("test 2", 10, CPU, 1)[0] is not small
    at = small.data_ptr()
    big, n = _lib._workspace("test", 1001, CPU, 1)
    assert n == big.numel() >= 2000
    del small
    assert at in {t.data_ptr() for t in _lib._ws.retired}
    assert _lib._workspace("test", 0, CPU, 1) == (None, 0)
