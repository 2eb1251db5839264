"""Every call of the norm, the convolution, the scan and beam search runs on
its own thread's stream, its workspace from there too (the library replaced by
one that only notes streams; no GPU)."""
import threading
import types

import pytest
import torch

from paper_1810_09958_gb300 import isam
from test_threads_cpu import Library, Tensor, b, f, u


class Serving(Library):
    def isam_rms_norm_backward_workspace(self, T, D, out):
        out._obj.value = 64
        return 0

    def isam_beam_select_workspace(self, batch, beams, V, count, out):
        out._obj.value = 64
        return 0


def i(n):
    return Tensor(n, torch.int32)


SSM = lambda n: (f(n * 4), f(n * 4), f(4), f(32), f(n * 8), f(n * 8), f(4), f(n * 4))
CALLS = {
    "rms_norm_forward": lambda: isam.rms_norm_forward(2, 8, f(16), b(16), b(16), f(8), 1e-5, b(16)),
    "rms_norm_forward_mx": lambda: isam.rms_norm_forward(2, 8, f(16), None, None, f(8), 1e-5, None, u(16), u(8)),
    "rms_norm_backward": lambda: isam.rms_norm_backward(2, 8, b(16), f(8), 1e-5, f(16), None, f(16), f(8), u(64)),
    "rms_norm_backward_own_workspace": lambda: isam.rms_norm_backward(2, 8, b(16), f(8), 1e-5, f(16), None, f(16), f(8)),
    "conv1d_forward": lambda: isam.conv1d_forward(3, 1, 4, 4, b(12), f(16), f(4), True, b(12), i(1), f(12), b(12)),
    "conv1d_step": lambda: isam.conv1d_step(1, 4, 4, 2, b(4), f(16), f(4), True, i(1), b(24), b(24), f(4)),
    "ssm_forward": lambda: isam.ssm_forward(3, 1, 4, 8, *SSM(3), f(32), i(1), f(12), f(32)),
    "ssm_step": lambda: isam.ssm_step(1, 4, 8, 2, *SSM(1), i(1), f(64), f(64), f(4)),
    "beam_select": lambda: isam.beam_select(1, 2, 9, 2, f(18), f(2), 3, u(2), f(2), i(2), i(2), u(2), u(64)),
    "beam_select_own_workspace": lambda: isam.beam_select(1, 2, 9, 2, f(18), f(2), 3, u(2), f(2), i(2), i(2), u(2)),
}


@pytest.mark.parametrize("name", CALLS)
def test_each_thread_runs_on_its_own_stream(name, monkeypatch):
    lib, mine, workspaces = Serving(), threading.local(), {}

    def alloc(size, stream):
        workspaces[threading.current_thread().name] = stream
        return 8192

    allocator = types.SimpleNamespace(_cuda_cudaCachingAllocator_raw_alloc=alloc,
                                      _cuda_cudaCachingAllocator_raw_delete=lambda at: None)
    monkeypatch.setattr(isam, "_torch", types.SimpleNamespace(float32=torch.float32, bfloat16=torch.bfloat16, int32=torch.int32,
                                                              uint8=torch.uint8, bool=torch.bool, _C=allocator))
    monkeypatch.setattr(isam, "_kinds", {torch.float32: 0, torch.bfloat16: 1})
    monkeypatch.setattr(isam, "_lib", lib)
    monkeypatch.setattr(isam, "_current_device", lambda: 0)
    monkeypatch.setattr(isam, "_raw_stream", lambda device: mine.stream)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    failed = []

    def work(stream):
        mine.stream = stream
        try:
            CALLS[name]()
        except Exception as e:  # (an exception in a thread does not fail a test by itself)
            failed.append(e)

    threads = {s: threading.Thread(target=work, args=(s,), name=f"stream {s}") for s in (1, 2)}
    for t in threads.values():
        t.start()
    for t in threads.values():
        t.join(30)
    assert not failed, failed
    assert lib.ran == {t.name: s for s, t in threads.items()}
    if name.endswith("own_workspace"):
        assert workspaces == lib.ran
