"""Which stream's memory the binding takes for a workspace that the caller leaves to it (no GPU)."""
import contextlib
import types

import pytest


@pytest.mark.parametrize("call", ["coded_encode_worker_mm", "coded_straggler_matmul"])
@pytest.mark.parametrize("given", [False, True])
def test_automatic_workspace_is_the_streams_own(lib, monkeypatch, call, given):
    """Memory of the current stream may still be in use by what waits there, and is handed out again to it as soon as
    the call returns: a call on another stream takes memory of that stream."""
    torch = pytest.importorskip("torch")
    current = [None]

    @contextlib.contextmanager
    def on(stream):
        current[0], before = stream, current[0]
        yield
        current[0] = before

    asked = []

    def workspace(code, A, X):
        asked.append(current[0])

    class Library:
        def __getattr__(self, name):
            return lambda *a: lib.CODED_OK

    side = types.SimpleNamespace(cuda_stream=7)
    code = types.SimpleNamespace(handle=None, n=5, k=3)
    A, X = torch.zeros((6, 4), dtype=torch.bfloat16), torch.zeros((4, 2), dtype=torch.bfloat16)
    Y, out = torch.zeros((5, 2, 2)), torch.zeros((6, 2))
    monkeypatch.setattr(lib, "worker_workspace", workspace)
    monkeypatch.setattr(lib, "lib", Library)
    monkeypatch.setattr(lib, "_stream", lambda stream=None: 7)
    monkeypatch.setattr(torch.cuda, "stream", on)
    stream = side if given else None
    if call == "coded_encode_worker_mm":
        lib.coded_encode_worker_mm(code, A, None, X, Y, stream=stream)
    else:
        lib.coded_straggler_matmul(code, A, None, X, Y, out, None, 0, 0, 1.0, stream=stream)
    assert asked == [stream] and current[0] is None
